// Stand-alone kernels (one per tile function), the kernels that repack weights at bind time, and the task table: which kernel
// a node gets, decided from its shapes.
#include "ng_kernels.hip"

namespace ng {
namespace {

// Batch-norm parameters -> one multiplier and one offset per channel, once, at bind time.
__global__ __launch_bounds__(kBlock) void fold_bn_kernel(const float* gamma, const float* beta, const float* mean,
                                                         const float* var, float eps, float* scale, float* shift, int C) {
    const int c = blockIdx.x * kBlock + threadIdx.x;
    if (c >= C) return;
    const float s = gamma[c] / sqrtf(var[c] + eps);
    scale[c] = s;
    shift[c] = beta[c] - mean[c] * s;
}

// The weights of both patch-stationary kernels, W[Cout][Cin][TAPS]: -> [block * TAPS + tap][Mf][part][lane][8 bf16], block = 16
// input channels, Mf = fragments of 32 rows; lane (r, g) holds row r, channels 8 g .. 8 g + 7; zero where m >= Cout.
// One thread per (slice, fragment, lane).
__global__ __launch_bounds__(kBlock) void pack_split_weights_kernel(const float* w, float* wq, int Cout, int Cin, int taps, int Mf, long total) {
    const long idx = (long)blockIdx.x * kBlock + threadIdx.x;
    if (idx >= total) return;
    const int lane = (int)(idx & 63);
    const long f = idx >> 6;
    const int mf = (int)(f % Mf), slice = (int)(f / Mf), block = slice / taps, tap = slice - block * taps;
    const int m = mf * 32 + (lane & 31), c = block * 16 + 8 * (lane >> 5);
    float v[8];
    for (int q = 0; q < 8; ++q) v[q] = m < Cout && c + q < Cin ? w[((size_t)m * Cin + c + q) * taps + tap] : 0.f;
    u32x4 part[3];
    split8(v, part);
    for (int p = 0; p < 3; ++p) reinterpret_cast<u32x4*>(wq)[(f * 3 + p) * 64 + lane] = part[p];
}

// W[Cout][Cin] -> W^T[CinP][CoutP], zero where k >= Cin or m >= Cout
__global__ __launch_bounds__(kBlock) void pack_pw_lds_weights_kernel(const float* w, float* wp, int Cout, int Cin, int CoutP, long total) {
    const long idx = (long)blockIdx.x * kBlock + threadIdx.x;
    if (idx >= total) return;
    const int m = (int)(idx % CoutP), k = (int)(idx / CoutP);
    wp[idx] = (m < Cout && k < Cin) ? w[(size_t)m * Cin + k] : 0.f;
}

// W[Cout][Cin][3][3] -> W'^T[tap * CinP + ci][CoutP], zero where ci >= Cin or m >= Cout
__global__ __launch_bounds__(kBlock) void pack_c3_lds_weights_kernel(const float* w, float* wp, int Cout, int Cin, int CinP, int CoutP, long total) {
    const long idx = (long)blockIdx.x * kBlock + threadIdx.x;
    if (idx >= total) return;
    const int m = (int)(idx % CoutP);
    const int k = (int)(idx / CoutP);
    const int tap = k / CinP, ci = k - tap * CinP;
    wp[idx] = (m < Cout && ci < Cin) ? w[((size_t)m * Cin + ci) * 9 + tap] : 0.f;
}

__global__ __launch_bounds__(kBlock) void pack_pw_weights_kernel(const float* w, float* wp, int Cout, int Cin,
                                                                  int ksteps, int total) {
    const int i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const int l = i & 63, blk = i >> 6;
    const int ks = blk % ksteps, rt = blk / ksteps;
    const int m = rt * 16 + (l & 15), k = ks * 4 + (l >> 4);
    wp[i] = (m < Cout && k < Cin) ? w[(size_t)m * Cin + k] : 0.f;
}

__global__ __launch_bounds__(kBlock) void pack_pw_weights_k4_kernel(const float* w, float* wp, int Cout, int Cin,
                                                                     int groups, int total) {
    const int i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const int q = i & 3, l = (i >> 2) & 63, blk = i >> 8;
    const int gi = blk % groups, rt = blk / groups;
    const int m = rt * 16 + (l & 15), k = 16 * gi + 4 * q + (l >> 4);
    wp[i] = (m < Cout && k < Cin) ? w[(size_t)m * Cin + k] : 0.f;
}
// Stand-alone kernel of one tile function: one workgroup per tile.
template <int KID>
__global__ __launch_bounds__(block_threads(KID), min_waves(KID)) void standalone_kernel(typename KernelOf<KID>::Args a) {
    __shared__ __align__(16) float smem[smem_floats(KID)];
    NoWait wait;
    KernelOf<KID>::template tile<false>(a, blockIdx.x, smem, threadIdx.x, true, wait);
}

// The same, with the device's clock read around it: workgroup b leaves in stamps[2 b] the time of its
// first instruction and in stamps[2 b + 1] the time at which all its stores were acknowledged (100 MHz
// constant clock; plain stores, one pair per workgroup, so the readings do not disturb each other). The
// latest end minus the earliest start is the time the GPU is busy with the task when it runs alone,
// without what the command processor spends around a dispatch.
template <int KID>
__global__ __launch_bounds__(block_threads(KID), min_waves(KID)) void timed_kernel(typename KernelOf<KID>::Args a, unsigned long long* stamps) {
    __shared__ __align__(16) float smem[smem_floats(KID)];
    unsigned long long t0 = 0;
    if (threadIdx.x == 0) t0 = wall_clock64();
    NoWait wait;
    KernelOf<KID>::template tile<false>(a, blockIdx.x, smem, threadIdx.x, true, wait);
    __builtin_amdgcn_s_waitcnt(0x0F70);                          // vmcnt(0): this wave's stores are acknowledged
    __syncthreads();
    if (threadIdx.x == 0) {
        stamps[2 * (size_t)blockIdx.x] = t0;
        stamps[2 * (size_t)blockIdx.x + 1] = wall_clock64();
    }
}

// ------------------------------------------------------------------------------------
// task construction
// ------------------------------------------------------------------------------------
template <int KID>
void set_kernel(Task& t, const typename KernelOf<KID>::Args& a, long ntiles) {
    using A = typename KernelOf<KID>::Args;
    static_assert(sizeof(A) <= kLaunchArgBytes, "argument block too large");
    static_assert(std::is_trivially_copyable<A>::value, "argument block must be plain data");
    t.kid = KID;
    t.fn = reinterpret_cast<const void*>(&standalone_kernel<KID>);
    t.name = KernelOf<KID>::name;
    std::memcpy(t.args, &a, sizeof(A));
    t.args_bytes = sizeof(A);
    t.ntiles = ntiles;
    t.grid[0] = (unsigned)ntiles;
    t.block[0] = block_threads(KID);
}

long ceil_div(long a, long b) { return (a + b - 1) / b; }

// conv1x1 forward / input gradient of a graph that trains: the kernel that reads pixels 128 bits at a time re-reads the
// activations once per 16 rows, which pays while the rows are few (the 64 x 64 LDS-staged GEMM tile otherwise).
bool pw_px_applies(const GemmArgs& a) {
    const long hw = (long)a.Ho * a.Wo;
    return hw >= 4 && a.K % 4 == 0 && a.M <= 256 && a.bias == nullptr && (long)a.K * a.N * 4 < (1L << 31) &&
           (long)a.M * a.N * 4 < (1L << 31);
}
// The classifier's GEMMs (1 x 1 maps, a few thousand outputs, K up to a few hundred): no tiles. K over the lanes of a
// wavefront where both operands run along k and K is long, else a thread per output.
constexpr long kSmallGemmOutputs = 1 << 16, kSmallGemmK = 1024;
void set_small_gemm(Task& t, SmallGemmArgs a, void (*set)(Task&, const SmallGemmArgs&, long)) {
    a.by_wave = a.sak == 1 && a.sbk == 1 && a.K >= 64;
    set(t, a, a.by_wave ? ceil_div((long)a.M * a.N, kBlock / 64) : ceil_div((long)a.M * a.N, kBlock));
}
long pw_px_tiles(const GemmArgs& a) {
    const long hw = (long)a.Ho * a.Wo;
    return ceil_div(ceil_div(a.N / hw * ceil_div(hw, 4), 16) * ceil_div(a.M, 16), 4);
}
// Backward kernels whose ragged edges (planes or rows that are no multiple of 16 or 4 pixels) cost extra work per edge: below
// this many pixels (weight gradients) or elements (depthwise input gradient) a task is a few workgroups that wait for
// memory once either way, and the general kernels stay. Above it, a training step of a NAS cell: 36 channels, 10 images of
// 27 x 27 pixels 1090 -> 750 us; 24 channels, 60 images of 30 x 30 pixels 2945 -> 1225 us.
constexpr long kRaggedMinPixels = 1024, kRaggedMinElements = 1 << 16;

// Direct conv1x1: k steps per chunk by problem depth, and the padded step count of the packed copy.
int pw_chunk(long cin) { return cin <= 64 ? 4 : (cin <= 128 ? 8 : 16); }
int pw_padded_steps(long cin) {
    const long unit = 4L * pw_chunk(cin);
    return (int)(ceil_div(ceil_div(cin, 4), unit) * unit);
}

}  // namespace

// Which XCD runs workgroup i? The planner relies on workgroups with equal i mod 8 sharing one
// (a 1-D grid is dealt out round-robin on this GPU); the runtime checks it with this probe
// before it trusts XCD-local L2s.
namespace {
__global__ __launch_bounds__(kGroup) void xcd_probe_kernel(int* xcd_of_workgroup) {
    if (threadIdx.x == 0) xcd_of_workgroup[blockIdx.x] = (int)__builtin_amdgcn_s_getreg(20 | (0 << 6) | (3 << 11));   // XCC_ID, bits 3:0
}
}  // namespace
const void* xcd_probe_kernel_handle() { return reinterpret_cast<const void*>(&xcd_probe_kernel); }

// Where the partial results of a weight-gradient task are (kind PARTS_NONE: it has none, it writes the gradient itself), and
// the same task with its sum left to a later launch.
SgdTile gradient_parts(const Task& t) {
    SgdTile p{};
    switch (t.kid) {
        case KID_GEMM_PW_WGRAD: case KID_GEMM_C3_WGRAD: case KID_PW_WGRAD_PX: case KID_PW_WGRAD_PX2: case KID_C3_WGRAD_PX: case KID_C3_WGRAD_PX2: {
            GemmArgs a;
            std::memcpy(&a, t.args, sizeof a);
            if (a.splits <= 1) break;
            p.kind = PARTS_BLOCKS, p.parts = a.ws, p.splits = a.splits, p.width = a.N, p.blocks = a.tiles_n;
            p.edge = (t.kid == KID_GEMM_PW_WGRAD || t.kid == KID_GEMM_C3_WGRAD) ? kGemmTile : (t.kid == KID_PW_WGRAD_PX || t.kid == KID_C3_WGRAD_PX) ? 16 : 32;
            break;
        }
        case KID_DW_WGRAD: {
            DwGradArgs a;
            std::memcpy(&a, t.args, sizeof a);
            if (a.chunks > 1) p.kind = PARTS_PLANES, p.parts = a.ws, p.splits = a.chunks, p.width = a.K * a.K;
            break;
        }
        case KID_BN_WGRAD: {
            BnRawArgs a;
            std::memcpy(&a, t.args, sizeof a);
            if (a.chunks > 1) p.kind = PARTS_PAIRS, p.parts = a.ws, p.splits = a.chunks, p.width = a.C;
            break;
        }
        default: break;
    }
    return p;
}
void leave_sum_to_later_launch(Task& t) {
    if (t.kid == KID_DW_WGRAD) reinterpret_cast<DwGradArgs*>(t.args)->cnt = nullptr;
    else if (t.kid == KID_BN_WGRAD) reinterpret_cast<BnRawArgs*>(t.args)->cnt = nullptr;
    else reinterpret_cast<GemmArgs*>(t.args)->cnt = nullptr;
}

// The launch that carries out the update nodes `members` (their stand-alone tasks in `tasks`) at once; in_parts[v] != 0:
// gradient node v is left in parts. The shares of the members are appended to `table`, the host copy of the device
// table that will sit at `table_dev`: the task's argument points at its first share there.
void make_sgd_batch_task(const ng_graph* g, const std::vector<Task>& tasks, const std::vector<int>& members, const std::vector<char>& in_parts,
                         std::vector<SgdTile>& table, const SgdTile* table_dev, Task& t) {
    const size_t first = table.size();
    for (int v : members) {
        SgdArgs a;
        std::memcpy(&a, tasks[v].args, sizeof a);
        const int gradient = g->nodes[v].preds[0];
        const bool parts = in_parts[gradient] != 0;
        const int per = parts ? kSgdSumElems : kSgdTileElems;
        for (int at = 0; at < a.total || at == 0; at += per) {
            SgdTile s = parts ? gradient_parts(tasks[gradient]) : SgdTile{};
            s.w = a.w + at, s.g = const_cast<float*>(a.g) + a.offset + at, s.flag = at == 0 ? a.flag : nullptr, s.lr = a.lr;
            s.count = std::min(a.total - at, per), s.first = a.offset + at;
            table.push_back(s);
        }
    }
    t = Task();
    t.block[0] = kBlock;
    set_kernel<KID_SGD_BATCH>(t, SgdBatchArgs{table_dev + first}, (long)(table.size() - first));
}

// Which two stand-alone kernels have a launch of their own together (pair_tile): input gradient first, weight gradient second.
static int pair_kid(const Task& first, const Task& second) {
    const int kid_first = first.kid, kid_second = second.kid;
    if (kid_first == KID_DW_DGRAD && kid_second == KID_DW_WGRAD) return KID_PAIR_DW;
    if (kid_first == KID_DW_DGRAD_LDS && kid_second == KID_DW_WGRAD)
        return dw_wgrad_by_quads(*reinterpret_cast<const DwGradArgs*>(second.args)) ? KID_PAIR_DW_LDS : KID_NONE;
    if (kid_first == KID_PW_PX_DGRAD && kid_second == KID_PW_WGRAD_PX) return KID_PAIR_PW16;
    if (kid_first == KID_PW_PX_DGRAD && kid_second == KID_PW_WGRAD_PX2) return KID_PAIR_PW32;
    if (kid_first == KID_ATTN_DK_T64 && kid_second == KID_ATTN_DV_T64) return KID_ATTN_DKV_T64;
    if (kid_first == KID_ATTNB_DK_T64 && kid_second == KID_ATTNB_DV_T64) return KID_ATTNB_DKV_T64;
    if (kid_first == KID_ATTNB_DQ_T64 && kid_second == KID_ATTNB_DB_T64) return KID_ATTNB_DQB_T64;
    if (kid_first == KID_ROPE_DX_4 && kid_second == KID_ROPE_DG_4) return KID_ROPE_BOTH_4;
    if (kid_first == KID_ROPE_DX_8 && kid_second == KID_ROPE_DG_8) return KID_ROPE_BOTH_8;
    if (kid_first == KID_ROPE_DX_N && kid_second == KID_ROPE_DG_N) return KID_ROPE_BOTH_N;
    if (kid_first == KID_NORM_DX_V8 && kid_second == KID_NORM_DG_V8) return KID_NORM_BOTH_V8;
    if (kid_first == KID_NORM_DX_H8 && kid_second == KID_NORM_DG_H8) return KID_NORM_BOTH_H8;
    if (kid_first == KID_NORM_DX_S16 && kid_second == KID_NORM_DG_S16) return KID_NORM_BOTH_S16;
    if (kid_first == KID_NORM_DX_M && kid_second == KID_NORM_DG_M) return KID_NORM_BOTH_M;
    if (kid_first == KID_NORM_DX_W8 && kid_second == KID_NORM_DG_W8) return KID_NORM_BOTH_W8;
    if (kid_first == KID_NORM_DX_W16 && kid_second == KID_NORM_DG_W16) return KID_NORM_BOTH_W16;
    return KID_NONE;
}
bool can_pair(const Task& first, const Task& second) {
    const int kid = pair_kid(first, second);
    if (!is_attention_tile_kernel(kid)) return kid != KID_NONE;
    AttnArgs a, b;                                             // its workgroups are cut in one way for both
    std::memcpy(&a, first.args, sizeof a);
    std::memcpy(&b, second.args, sizeof b);
    return a.col_blocks == b.col_blocks && a.splits == b.splits && a.per_split == b.per_split;
}
// The kernel of the launch of task v with everything that rides on it (`fused_into` as decided).
int launch_kid(const std::vector<Task>& tasks, const std::vector<int>& fused_into, int v) {
    for (size_t w = 0; w < tasks.size(); ++w) {
        if (fused_into[w] != v || (int)w == v) continue;
        const int a = tasks[v].kid, b = tasks[w].kid;
        if (b == KID_SGD) return KID_SGD_BATCH;
        if ((a == KID_BN_DGRAD && b == KID_BN_WGRAD) || (a == KID_BN_WGRAD && b == KID_BN_DGRAD)) return KID_BN_BACKWARD;
        if (can_pair(tasks[v], tasks[w])) return pair_kid(tasks[v], tasks[w]);
        if (can_pair(tasks[w], tasks[v])) return pair_kid(tasks[w], tasks[v]);
    }
    return tasks[v].kid;
}
template <int KID>
static void set_pair(const Task& first, const Task& second, Task& t) {
    typename KernelOf<KID>::Args p{};
    std::memcpy(&p.a, first.args, sizeof p.a);
    std::memcpy(&p.b, second.args, sizeof p.b);
    p.na = (int)first.ntiles, p.nb = (int)second.ntiles;
    t = Task();
    t.block[0] = kBlock;
    set_kernel<KID>(t, p, first.ntiles + second.ntiles);
}
template <int KID>
static void set_pw_backward(const Task& dgrad, const Task& wgrad, Task& t) {
    PairPwArgs p{};
    std::memcpy(&p.a, dgrad.args, sizeof p.a);
    std::memcpy(&p.b, wgrad.args, sizeof p.b);
    const long hw = (long)p.a.Ho * p.a.Wo, groups = ceil_div(p.a.N / hw * ceil_div(hw, 4), 16);
    p.na = (int)ceil_div((p.b.splits >= kXcdSplits ? ceil_div(groups, p.b.splits) : groups) * ceil_div(p.a.M, 16), 4);
    p.nb = (int)(wgrad.ntiles / p.b.splits);
    t = Task();
    t.block[0] = kBlock;
    set_kernel<KID>(t, p, pw_backward_tiles(p.na, p.nb, p.b.splits));
}
// Both gradients of norm and rotation, or of a layer norm: the walk of the weight gradient, whose workgroups leave rows of sums, with dx
// written on the way.
template <int KID>
static void set_norm_backward(const Task& dgrad, const Task& wgrad, Task& t) {
    typename KernelOf<KID>::Args a, d;
    std::memcpy(&a, wgrad.args, sizeof a);
    std::memcpy(&d, dgrad.args, sizeof d);
    a.y = d.y;
    t = Task();
    t.block[0] = kBlock;
    set_kernel<KID>(t, a, wgrad.ntiles);
}
// dq's task with the result and the rows of sums of the bias's gradient.
template <int KID>
static void set_dq_dbias(const Task& dq, const Task& dbias, Task& t) {
    AttnArgs a, b;
    std::memcpy(&a, dq.args, sizeof a);
    std::memcpy(&b, dbias.args, sizeof b);
    a.db = b.db, a.db_ws = b.db_ws, a.db_cnt = b.db_cnt;
    t = Task();
    t.block[0] = kBlock;
    set_kernel<KID>(t, a, dq.ntiles);
}
void make_pair_task(const Task& first, const Task& second, Task& t) {
    switch (pair_kid(first, second)) {
        case KID_PAIR_DW: set_pair<KID_PAIR_DW>(first, second, t); break;
        case KID_PAIR_DW_LDS: set_pair<KID_PAIR_DW_LDS>(first, second, t); break;
        case KID_PAIR_PW16: set_pw_backward<KID_PAIR_PW16>(first, second, t); break;
        case KID_PAIR_PW32: set_pw_backward<KID_PAIR_PW32>(first, second, t); break;
        case KID_ATTN_DKV_T64:                                  // the same workgroups for both
            set_pair<KID_ATTN_DKV_T64>(first, second, t);
            t.ntiles = first.ntiles, t.grid[0] = (unsigned)first.ntiles;
            break;
        case KID_ATTNB_DKV_T64:
            set_pair<KID_ATTNB_DKV_T64>(first, second, t);
            t.ntiles = first.ntiles, t.grid[0] = (unsigned)first.ntiles;
            break;
        case KID_ATTNB_DQB_T64: set_dq_dbias<KID_ATTNB_DQB_T64>(first, second, t); break;
        case KID_ROPE_BOTH_4: set_norm_backward<KID_ROPE_BOTH_4>(first, second, t); break;
        case KID_ROPE_BOTH_8: set_norm_backward<KID_ROPE_BOTH_8>(first, second, t); break;
        case KID_ROPE_BOTH_N: set_norm_backward<KID_ROPE_BOTH_N>(first, second, t); break;
        case KID_NORM_BOTH_V8: set_norm_backward<KID_NORM_BOTH_V8>(first, second, t); break;
        case KID_NORM_BOTH_H8: set_norm_backward<KID_NORM_BOTH_H8>(first, second, t); break;
        case KID_NORM_BOTH_S16: set_norm_backward<KID_NORM_BOTH_S16>(first, second, t); break;
        case KID_NORM_BOTH_M: set_norm_backward<KID_NORM_BOTH_M>(first, second, t); break;
        case KID_NORM_BOTH_W8: set_norm_backward<KID_NORM_BOTH_W8>(first, second, t); break;
        case KID_NORM_BOTH_W16: set_norm_backward<KID_NORM_BOTH_W16>(first, second, t); break;
        default: t = first; break;
    }
}

// The launch that computes a batch-norm's parameter gradients (task `wgrad`) and its input gradient (task `dgrad`, same
// dy, x and parameters) in one walk over dy and x.
void make_bn_backward_task(const Task& dgrad, const Task& wgrad, Task& t) {
    BnRawArgs a, d;
    std::memcpy(&a, wgrad.args, sizeof a);
    std::memcpy(&d, dgrad.args, sizeof d);
    a.dx = d.y;
    t = Task();
    t.block[0] = kBlock;
    set_kernel<KID_BN_BACKWARD>(t, a, wgrad.ntiles);
}

template <> const void* resident_build_handle<BUILD_LEAN>();
template <> const void* resident_build_handle<BUILD_FULL>();
template <> const void* resident_build_handle<BUILD_TRAIN>();
template <> const void* resident_build_handle<BUILD_ATTENTION>();
const void* resident_kernel_handle(int build) {
    return build == BUILD_ATTENTION ? resident_build_handle<BUILD_ATTENTION>() : build == BUILD_TRAIN ? resident_build_handle<BUILD_TRAIN>() : build == BUILD_FULL ? resident_build_handle<BUILD_FULL>() : resident_build_handle<BUILD_LEAN>();
}

namespace {
__global__ void empty_kernel() {}
}  // namespace
const void* empty_kernel_handle() { return reinterpret_cast<const void*>(&empty_kernel); }

// The stand-alone kernel of a kernel id (nullptr if the id has none) and its name: lets the runtime
// launch a task in the variant a replay mode really executes (e.g. a convolution with its fused
// batch-norm and add_n), by itself, for timing.
const void* standalone_kernel_handle(int kid, const char** name) {
    switch (kid) {
#define NG_HANDLE(KID) \
    case KID:          \
        if (name) *name = KernelOf<KID>::name; \
        return reinterpret_cast<const void*>(&standalone_kernel<KID>);
        NG_FOR_EACH_KID(NG_HANDLE)
#undef NG_HANDLE
        default: return nullptr;
    }
}
const void* timed_kernel_handle(int kid) {
    switch (kid) {
#define NG_HANDLE(KID) \
    case KID: return reinterpret_cast<const void*>(&timed_kernel<KID>);
        NG_FOR_EACH_KID(NG_HANDLE)
#undef NG_HANDLE
        default: return nullptr;
    }
}

namespace {
// Which conv1x1 kernel a node gets. Decided from shapes alone, so that the size of the
// repacked weights is known before any memory is bound.
struct PwChoice {
    enum Kind { NONE, GEMV, LDS64, DIRECT32, K4_VEC, K4_WORD, C3_LDS, C3_PATCH, PW_PATCH } kind = NONE;
    int kid = KID_NONE;       // C3_PATCH, PW_PATCH: which of the kernels
    int in_flight = 0;        // K4: groups of 4 k-steps in flight (1..4); DIRECT32: k-steps per chunk
    int groups = 0;           // K4: groups in the packed copy (a multiple of 4 * in_flight); DIRECT32: padded k-steps
    size_t packed = 0;        // floats of repacked weights
};
// K split of the 16-row kernels: groups of 4 k-steps, padded so that every wavefront gets
// the same whole number of chunks of `in_flight` groups.
void k4_split(long k_total, long cout, PwChoice& c) {
    const long groups = ceil_div(ceil_div(k_total, 4), 4);
    long gw = ceil_div(groups, 4);                           // groups per wavefront
    if (gw <= 4) {
        c.in_flight = (int)gw;
    } else {
        const long pad3 = ceil_div(gw, 3) * 3, pad4 = ceil_div(gw, 4) * 4;
        c.in_flight = pad3 < pad4 ? 3 : 4;
        gw = std::min(pad3, pad4);
    }
    c.groups = (int)(4 * gw);
    c.packed = (size_t)((cout + 15) / 16) * c.groups * 256;
}
constexpr long kPwPatchMinCols = 2048;
constexpr long kPoolRowMinOutputs = 1 << 20;   // pool3x3: from here on the kernel with four outputs of a column per thread
constexpr long kDwLdsMinOutputs = 1 << 18;     // dwconv: from here on whole planes through LDS (dwconv_lds), where the planes allow
PwChoice choose_pw(const ng_graph* g, int v) {
    PwChoice c;
    const Node& nd = g->nodes[v];
    if (nd.op != NG_OP_CONV1X1 && nd.op != NG_OP_FC) return c;
    const Shape& o = nd.out;
    const long cin = g->nodes[nd.preds[0]].out.c;
    const long hw = o.h * o.w, cols = o.n * hw;
    if (nd.op == NG_OP_FC && o.n <= 8) { c.kind = PwChoice::GEMV; return c; }
    // many output pixels, whole blocks of 16 input channels: activations pixel-major in LDS, weights straight from memory;
    // 64-row tiles unless that leaves most compute units without one
    const long tiles64 = ((o.c + 63) / 64) * ((cols + 63) / 64);
    if (cols >= kPwPatchMinCols && cin % 16 == 0 && cin >= 64 && tiles64 >= 64 && cols * cin * 4 < (1L << 31) && cin * (o.c + 63) * 6 < (1L << 31) && !knob("NG_NO_PATCH_KERNELS")) {
        c.kind = PwChoice::PW_PATCH;
        c.kid = tiles64 < 200 ? KID_PW_P32 : KID_PW_P64;
        const long tm = c.kid == KID_PW_P32 ? 32 : 64;
        c.groups = (int)cin;
        c.packed = (size_t)cin * (size_t)((o.c + tm - 1) / tm * tm) * 3 / 2;   // [Cin / 16][CoutP / 32][3 parts][64 lanes][8 bf16]
        return c;
    }
    // large problems (many 64 x 64 tiles) keep the LDS-tiled throughput kernel
    if (((o.c + 63) / 64) * ((cols + 63) / 64) >= 256) {
        c.kind = PwChoice::LDS64;
        c.groups = (int)((cin + 15) / 16 * 16);                              // CinP: whole K slices of 16
        c.packed = (size_t)c.groups * (size_t)((o.c + 63) / 64 * 64);       // W^T[CinP][CoutP]
        return c;
    }
    const bool vec = hw % 4 == 0;
    const long tiles16 = ((o.c + 15) / 16) * ((cols + 15) / 16);
    // Maps without 128-bit loads: the 16 x 16 tiles with K split over the wavefronts up to 512 of them (two workgroups per
    // compute unit), 32 x 32 tiles, which read less, beyond. The 32 x 32 kernels hold registers that only the full build of
    // the resident kernel has room for: a NAS cell on 25 x 25 maps (240 tiles) replays in 356 us with 16 x 16 tiles (lean
    // build) and in 474 us with two of its tasks on 32 x 32 tiles, which take 4.2 us there against 2.9 us; an
    // Inception-style network at batch 1 (31 layers of 17 x 17 and 35 x 35 maps, 228 - 385 tiles) 765 against 810 us.
    // Graphs in the full build and launched ones gain as well: of chains of twelve layers between 44 - 2048 channels, 7 x 7 to 45 x 45
    // (121 - 512 tiles), 17 of 17 are faster as a single-stream graph and 15 in the resident kernel (two 2 % slower): 17 x 17 768 <-> 192 86 / 175 -> 63 / 123 us, 35 x 35
    // 64 <-> 64 46 / 80 -> 42 / 46, 7 x 7 2048 <-> 1000 162 / 350 -> 103 / 115, 35 x 35 1024 <-> 64 120 / 197 -> 113 / 183.
    if (!vec && tiles16 > 512) {
        c.kind = PwChoice::DIRECT32;
        c.in_flight = pw_chunk(cin);
        c.groups = pw_padded_steps(cin);
        c.packed = (size_t)((o.c + 15) / 16) * 64 * c.groups;
        return c;
    }
    c.kind = vec ? PwChoice::K4_VEC : PwChoice::K4_WORD;
    k4_split(cin, o.c, c);
    return c;
}
// conv3x3 with at least 8 input channels runs as an implicit GEMM with K = 9 Cin
constexpr long kC3LdsMinCols = 2048;      // measured: below this the 16 x 16 tiles (more workgroups, shorter K loops each) win
// The patch-stationary kernels: rows and pixels of a tile; a tile's time while the chip is full of them (64: one of 64 x 64), from 430
// layers of 9 x 9 to 130 x 130, 16 - 384 output channels, strides of 1 and 2: choose_patch_kernel takes the fastest of the kernels, or one
// within 5 % of it.
struct PatchKernel { int kid, tm, tn; double cost; };
constexpr PatchKernel kPatchKernels[] = {{KID_C3_P64, 64, 64, 64}, {KID_C3_P96, 96, 64, 94}, {KID_C3_Q32, 32, 128, 68},
                                         {KID_C3_Q64, 64, 64, 73}, {KID_C3_Q128, 64, 128, 117}, {KID_C3_R32, 32, 128, 74},
                                         {KID_C3_R128, 64, 128, 140}, {KID_C3_SK, 32, 32, 0}};
// Largest patch a run of tn consecutive output pixels can need: the rows it touches (a run can start at the end of a
// row), stride apart, plus two, each W + 2 pad wide.
long patch_pixels(long tn, long W, long Ho, long Wo, long stride, long pad) {
    const long rows = std::min(Ho, (tn - 2) / Wo + 2);
    return ((rows - 1) * stride + 3) * (W + 2 * pad);
}
// The strips that an image is cut into, so that the patch of every run of tn pixels of a strip fits into the kernel's LDS: the width
// of all but the last (0: none fits) and the runs of an image. As few strips as possible, unless more of them save more than one run in 33.
struct Strips { long width, runs; };
long largest_patch(long tn, long width, long Ho, long stride) {              // as the kernel counts it, over the runs of one strip
    long most = 0;
    const long row = (width - 1) * stride + 3, pixels = width * Ho;
    auto run = [&](long p) {
        const long last = std::min(p + tn, pixels) - 1;
        most = std::max(most, ((last / width - p / width) * stride + 2) * row + last % width * stride + 3 - p % width * stride);
    };
    // a whole run's patch depends on the column it starts in, and those repeat after at most `width` runs; the last run may be short
    for (long i = 0, start = 0; i < width && start < pixels; ++i, start += tn) run(start);
    run((pixels - 1) / tn * tn);
    return most;
}
Strips choose_strips(int kid, long tn, long Ho, long Wo, long stride) {
    const long room = c3_patch_pixels(kid);
    auto fits = [&](long width) { return largest_patch(tn, width, Ho, stride) <= room; };
    const long widest = (room - 2 * 3 - 3) / 2 / stride + 1;                 // the smallest patch: two rows of the strip and three pixels
    Strips best{0, 0};
    for (long n = ceil_div(Wo, widest); n <= Wo; ++n) {
        const long width = ceil_div(Wo, n), rest = Wo - (ceil_div(Wo, width) - 1) * width;
        if (ceil_div(Wo, width) != n) continue;                               // the same width as with fewer strips
        if (!fits(width) || !fits(rest)) continue;
        const long runs = (n - 1) * ceil_div(width * Ho, tn) + ceil_div(rest * Ho, tn);
        if (best.width == 0 || runs * 33 < best.runs * 32) best = Strips{width, runs};
    }
    return best;
}
// whole blocks of 16 channels; activations and packed weights (three 16-bit parts) within the reach of a buffer descriptor
bool patch_reaches(const Shape& in, const Shape& out) {
    return in.c % 16 == 0 && in.n * in.c * in.h * in.w * 4 < (1L << 31) && 9 * in.c * (out.c + 95) * 6 < (1L << 31);
}
// Which patch kernel a conv3x3 gets (KID_NONE: none fits). Decided from shapes: a compute unit works its workgroups off side by
// side, so the estimate is (tiles per compute unit, rounded up) x a tile's time. One lone workgroup per compute unit cannot keep the
// matrix cores busy on its own: x 1.15, and x 1.25 for 64 x 128 over one or two blocks of channels, mostly filling patches (13 layers of 32
// channels: two rounds of 64 x 64 take 10.6 - 10.9 us there and one of 64 x 128 10.9 - 11.2; with 48 channels 13.2 and 12.6).
// Tiles are the runs of the strips: narrow strips have short runs, which count in full. 128 images of 64 x 33 x 33 to 384 channels,
// stride 2: 64 x 128 with 256 pixels of patch has six runs instead of two and takes 222 us; 64 x 64 takes 119, 64 x 128 with 640 pixels 93.
// The kernels for narrow images take images whose patches hold rows of whole width. Those with 640 pixels take only strides of 2 (at a
// stride of 1 32 x 128 takes 19.8 - 62 us, with 256 pixels 15.3 - 50), 32 x 128 with 256 only strides of 1 (2: 16 images of
// 64 x 45 x 45 -> 32 17.3 us, 64 x 64 with 384 13.1). The others take any width (4 images of 64 channels, stride 1, LDS-staged GEMM / now:
// 159 x 159 -> 32 66 / 30 us, 224 x 224 -> 64 161 / 72, 300 x 300 -> 96 527 / 210; 16 images, stride 2: 90 x 90 -> 64 35 / 25,
// 127 x 127 -> 32 54 / 23, 200 x 200 -> 192 405 / 225).
int choose_patch_kernel(const Shape& in, const Shape& out, long stride, long pad) {
    if (!patch_reaches(in, out)) return KID_NONE;
    int best = KID_NONE;
    double best_cost = 0;
    for (const PatchKernel& k : kPatchKernels) {
        const bool narrow = k.kid == KID_C3_P64 || k.kid == KID_C3_P96;
        if (k.kid == KID_C3_SK || (narrow && patch_pixels(k.tn, in.w, out.h, out.w, stride, pad) > c3_patch_pixels(k.kid))) continue;
        if ((k.tm == 32 && out.c > 32) || (stride == 1 ? c3_patch_pixels(k.kid) == 640 : k.kid == KID_C3_Q32)) continue;
        const Strips strips = choose_strips(k.kid, k.tn, out.h, out.w, stride);
        if (strips.width == 0) continue;
        const long rounds = ceil_div(out.n * strips.runs * ceil_div(out.c, k.tm), 256);
        const double lone = k.tm == 64 && k.tn == 128 && in.c <= 32 ? 1.25 : 1.15;
        const double cost = (double)rounds * k.cost * (rounds == 1 ? lone : 1.0);
        if (best == KID_NONE || cost < best_cost) best = k.kid, best_cost = cost;
    }
    return best;
}
PwChoice choose_c3(const ng_graph* g, int v) {
    PwChoice c;
    const Node& nd = g->nodes[v];
    if (nd.op != NG_OP_CONV3X3) return c;
    const Shape& in = g->nodes[nd.preds[0]].out;
    const long cin = in.c;
    if (cin < 8) return c;
    // The patch-stationary kernels. Few tiles of 64 x 64 (up to two for three compute units) leave the chip idle: 32 x 32 tiles
    // with K over the wavefronts, where the patches are small enough and every wavefront gets a block of 16 channels (with 32
    // channels 5.3 us against 4.1 of the gathering kernel). Us alone, gathering kernel / 64 x 64 tiles / these, tiles of 64 x 64:
    // 17 x 17 192 -> 192 one image 11.5 / 20.9 / 9.2 (15), 14 x 14 192 -> 192 six images 31 / 20 / 10 (72), 35 x 35 96 -> 96
    // four images 34 / 13.4 / 11.3 (160); 30 x 30 64 -> 96 six images 22.6 / 11.0 / 11.8 (180), 8 x 8 384 -> 768 twenty images
    // 196 / 41.5 / 43 (240). Where they don't apply (a stride of 2), from 96 tiles of 64 x 64 on the large tiles: 30 x 30 ->
    // 14 x 14 288 -> 384 six images 80 / 47 (144), one image of 35 x 35 -> 17 x 17 27 / 46 (30). 22 more layers of 64 - 512 channels
    // around the first line, 64 x 64 tiles / these: 120 - 144 tiles 10.3 - 53 / 7.4 - 30.4 (six, these 20 - 45 % faster), 156 - 160
    // 10.6 - 23.9 / 10.6 - 21.5, 180 - 192 10.5 - 52.5 / 10.7 - 40.6, 200 - 250 10.9 - 22.6 / 12.9 - 25.0 (these 9 - 33 % slower). Alone
    // these still win up to three 32 x 32 tiles on a compute unit (27 layers 0.73 - 0.99 of the time, one 1.06); but siblings share launches, which
    // fill the chip with large tiles: with that line the Inception-style network on six images takes 1058 us instead of 1026. 14 more
    // with a stride of 2 around the second, gathering kernel / 64 x 64: 48 tiles 35 / 44.5, 60 - 96 within 7 % of each other, 108
    // 26 / 18 and 67 / 47.5.
    if (!knob("NG_NO_PATCH_KERNELS")) {
        const long tiles64 = nd.out.n * ceil_div(nd.out.h * nd.out.w, 64) * ceil_div(nd.out.c, 64);
        int kid = choose_patch_kernel(in, nd.out, nd.p.stride, nd.p.pad);
        if (patch_reaches(in, nd.out) && cin >= 64 && tiles64 <= 170 && patch_pixels(32, in.w, nd.out.h, nd.out.w, nd.p.stride, nd.p.pad) <= c3_patch_pixels(KID_C3_SK))
            kid = KID_C3_SK;
        else if (nd.out.n * nd.out.h * nd.out.w < kC3LdsMinCols && (cin < 64 || tiles64 < 96))
            kid = KID_NONE;
        for (const PatchKernel& k : kPatchKernels)
            if (k.kid == kid) {
                c.kind = PwChoice::C3_PATCH, c.kid = kid;
                c.groups = (int)cin;                                                             // CinP = Cin (a multiple of 16)
                c.packed = (size_t)(9 * cin) * (size_t)(ceil_div(nd.out.c, k.tm) * k.tm) * 3 / 2;    // [9 Cin / 16][CoutP / 32][3 parts][64 lanes][8 bf16]
                return c;
            }
    }
    if (nd.out.n * nd.out.h * nd.out.w >= kC3LdsMinCols) {
        c.kind = PwChoice::C3_LDS;
        const long kc = nd.out.c <= 32 ? 16 : 32, tm = nd.out.c <= 32 ? 32 : 64;     // K slice and rows per tile of the two kernels
        c.groups = (int)((cin + kc - 1) / kc * kc);                                    // CinP
        c.packed = (size_t)(9 * c.groups) * (size_t)((nd.out.c + tm - 1) / tm * tm);  // W'^T[9 CinP][CoutP]
        return c;
    }
    c.kind = PwChoice::K4_WORD;
    k4_split(9 * cin, nd.out.c, c);
    return c;
}

}  // namespace

// Floats of library-owned constant memory node v needs (repacked conv1x1 weights), 0 if none.
namespace {
// K split of a weight-gradient GEMM: enough workgroups to occupy the GPU, splits of whole K slices
void gemm_split(long m, long n, long k, int* splits, int* k_per_split) {
    const long tiles = ceil_div(m, kGemmTile) * ceil_div(n, kGemmTile);
    // A split costs its share of the K slices (about 0.5 us each) and adds one partial tile to what the workgroup
    // that arrives last has to add up (about 0.4 us each): the sum is smallest near sqrt(1.25 x slices) splits.
    const double slices = (double)ceil_div(k, 16);
    long want = (long)std::lround(std::sqrt(1.25 * slices));
    want = std::max<long>(1, std::min<long>(want, std::max<long>(1, 768 / tiles)));
    const long per = ceil_div(ceil_div(k, want), 16) * 16;
    *k_per_split = (int)per;
    *splits = (int)ceil_div(k, per);
}
// geometry of a weight-gradient node: (M, N, K) of dW[M x N] = dY[M x K] * P^T[K x N]
bool wgrad_dims(const ng_graph* g, int v, long* m, long* n, long* k) {
    const Node& nd = g->nodes[v];
    if (nd.op != NG_OP_CONV1X1_WGRAD && nd.op != NG_OP_CONV3X3_WGRAD) return false;
    const Shape& dy = g->nodes[nd.preds[0]].out;
    const Shape& x = g->nodes[nd.preds[1]].out;
    *m = dy.c, *n = x.c * (nd.op == NG_OP_CONV3X3_WGRAD ? 9 : 1), *k = dy.n * dy.h * dy.w;
    return true;
}
// Workgroups a channel of a batch-norm or depthwise parameter gradient is split over (by images): about 512 workgroups in all
long bn_wgrad_chunks(long channels, long images, long workgroups = 512) {
    const long want = std::max<long>(1, std::min<long>(images, ceil_div(workgroups, channels)));
    return ceil_div(images, ceil_div(images, want));            // no empty chunk
}
long dw_wgrad_chunks(long channels, long images) { return bn_wgrad_chunks(channels, images, knob_int("NG_DW_WGRAD_WGS", 1, 4096, 512)); }
// How a weight-gradient node is computed: which kernel, how K is split, what workspace it needs.
struct WgradPlan {
    bool px = false;              // conv1x1_wgrad_px (both operands 128 bits along the pixels) instead of the gather GEMM
    bool small = false;           // small_gemm: 1 x 1 maps and a few thousand weights (the classifier), no split, no workspace
    int block = 0;                // px: fragments of 16 x 16 weights along each side of a workgroup's block (1 or 2)
    long tiles = 0;
    int splits = 1, k_per_split = 0;
    size_t ws_floats = 0;         // partial tiles (and group sums)
    size_t cnt_words = 0;         // arrival counters behind them, a multiple of 64
};
WgradPlan wgrad_plan(const ng_graph* g, int v) {
    WgradPlan p;
    long m, n, k;
    if (!wgrad_dims(g, v, &m, &n, &k)) return p;
    const Node& nd = g->nodes[v];
    const Shape& dy = g->nodes[nd.preds[0]].out;
    const Shape& x = g->nodes[nd.preds[1]].out;
    p.tiles = ceil_div(m, kGemmTile) * ceil_div(n, kGemmTile);
    const size_t tile_floats = (size_t)kGemmTile * kGemmTile;
    if (nd.op == NG_OP_CONV1X1_WGRAD && dy.h * dy.w == 1 && m * n <= kSmallGemmOutputs && k <= kSmallGemmK) {
        p.small = true, p.splits = 1, p.k_per_split = (int)k;
        return p;
    }
    const long hw = dy.h * dy.w;
    const bool c3 = nd.op == NG_OP_CONV3X3_WGRAD, whole = c3 ? dy.w % 16 == 0 : hw % 16 == 0;
    p.px = hw >= 4 && (whole || k >= kRaggedMinPixels) && dy.elems() * 4 < (1L << 31) && x.elems() * 4 < (1L << 31) &&
           (!c3 || (nd.p.stride == 1 && nd.p.pad == 1 && dy.w >= 4 && dy.h == x.h && dy.w == x.w));
    k = dy.n * ceil_div(hw, 16) * 16;                           // an image is a whole number of slices of 16 pixels
    const long fm = ceil_div(m, 16), fn = ceil_div(n, 16);
    p.px = p.px && fm * fn <= 256;
    if (p.px) {
        // Blocks of B x B fragments of 16 x 16 weights, each split over K: 512 pixels a split (eight slices of 16 for each of
        // the four wavefronts: one batch of loads) up to 128 splits, which somebody has to add up; where that leaves compute
        // units idle, 256 pixels for about two workgroups each. Training step of a NAS cell with 44 channels on 32 x 32
        // maps: batch 32 (64 splits) 1072 us, with 128 splits 1097; batch 96 (128 splits) 2187 us, with 64 splits 2220 -
        // 2230, with 32 splits 2266.
        p.block = fm * fn <= 16 ? 1 : 2;
        p.tiles = ceil_div(fm, p.block) * ceil_div(fn, p.block);
        const long most = 128;
        const long want = std::max<long>({1, std::min(k / 512, most), std::min<long>({ceil_div(k, 256), 512 / p.tiles, 64})});
        // of the splits near that (each a multiple of 64 pixels) the one whose XCDs, which take every eighth split, are
        // busiest for the shortest time
        long best = -1;
        for (long per = ceil_div(ceil_div(k, std::min(want * 5 / 4, most)), 64); per <= ceil_div(ceil_div(k, std::max<long>(1, want * 3 / 4)), 64); ++per) {
            const long cost = ceil_div(ceil_div(k, per * 64), 8) * per;
            if (best < 0 || cost < best) best = cost, p.k_per_split = (int)(per * 64);
        }
        p.splits = (int)ceil_div(k, p.k_per_split);
        if (p.splits > 1) {
            p.ws_floats = (size_t)p.tiles * p.splits * 256 * p.block * p.block;
            p.cnt_words = ((size_t)p.tiles + 63) & ~(size_t)63;
        }
        return p;
    }
    gemm_split(m, n, dy.n * hw, &p.splits, &p.k_per_split);
    if (p.splits > 1) {
        p.ws_floats = (size_t)p.tiles * p.splits * tile_floats;
        p.cnt_words = ((size_t)p.tiles + 63) & ~(size_t)63;
    }
    return p;
}
// How an attention node is computed: kernel, how the work is cut, and its share of the library-owned memory: workspace, then
// arrival counters, then (forward, if somebody reads them) two numbers of every query.
long round64(long n) { return (n + 63) & ~63L; }
struct AttentionPlan {
    int kid = KID_NONE;
    int col_blocks = 1, splits = 1, per_split = 1, query_blocks = 1;
    long tiles = 0;
    size_t ws_floats = 0, cnt_words = 0, stats_floats = 0;
};
bool is_attention_op(int op) { return (op >= NG_OP_ATTENTION && op <= NG_OP_ATTENTION_DV) || op == NG_OP_ATTENTION_DBIAS; }
// Splits of a tile kernel's other side: the number with which the task is expected to end first. A compute unit has two workgroups at a
// time, which take longer than one alone, but not twice as long; a last one that is left over has it to itself. A split costs what the
// workgroup that joins them reads. us, of the straight lines through what these kernels take with 1 .. 32 splits: 47 queries of 28 heads
// of 128 channels, 9950 keys, 6 splits 127, 8 102, 16 92, 24 128; dq of 175 queries of 120 heads on 30, 660 keys, 1 100, 2 78, 3 95, 8 98; dk of
// 93 keys of 13 heads of 96, 6892 queries each, 8 127, 16 80, 32 86.
long tile_splits(int op, bool narrow, long groups, long blocks) {
    const bool by_keys = op == NG_OP_ATTENTION_DK || op == NG_OP_ATTENTION_DV, both = by_keys && narrow;      // both: one launch, cut alike
    const bool heavy = !narrow && (op == NG_OP_ATTENTION_DQ || op == NG_OP_ATTENTION_DBIAS || op == NG_OP_ATTENTION_DK);
    const double one = heavy ? 4.4 : both ? 3.4 : 2.0;             // a block of a workgroup that is alone
    const double pair = heavy ? 5.8 : both ? 4.4 : narrow ? 2.5 : 3.2;      // of two
    const double around = heavy ? 8.0 : 6.0;                       // first loads, results
    const double join = both ? 8.0 : op == NG_OP_ATTENTION ? 6.0 : 4.0, join_each = both ? 1.1 : narrow ? 0.4 : op == NG_OP_ATTENTION ? 0.8 : 0.6;
    long best = 1;
    double least = 0;
    for (long want = 1; want <= std::min<long>(blocks, kMaxSplits); ++want) {
        const long each = ceil_div(blocks, want), splits = ceil_div(blocks, each), turns = ceil_div(groups * splits, 256);
        const double us = (double)(turns / 2) * ((double)each * pair + around) + (double)(turns % 2) * ((double)each * one + around) +
                          (splits > 1 ? join + join_each * (double)splits : 0.0);
        if (want == 1 || us < least) best = want, least = us;
    }
    return best;
}

AttentionPlan attention_plan(const ng_graph* g, int v) {
    AttentionPlan p;
    const Node& nd = g->nodes[v];
    if (!is_attention_op(nd.op) || nd.op == NG_OP_ATTENTION_ROWS) return p;
    const int first = nd.op == NG_OP_ATTENTION ? 0 : 2;
    const Shape &q = g->nodes[nd.preds[first]].out, &k = g->nodes[nd.preds[first + 1]].out;
    const long d = q.c / nd.p.heads, group = nd.p.heads / nd.p.kv_heads, Tq = q.h * q.w, Tk = k.h * k.w;
    const bool by_keys = nd.op == NG_OP_ATTENTION_DK || nd.op == NG_OP_ATTENTION_DV;
    const bool narrow = d <= 64;
    const bool biased = nd.p.bias != 0, dbias = nd.op == NG_OP_ATTENTION_DBIAS;
    // the kernels for heads of up to 64 channels; the next id: up to 128
    const int of_op = nd.op == NG_OP_ATTENTION ? 0 : dbias ? 4 : nd.op - NG_OP_ATTENTION_DQ + 1;
    const int waves[2][5] = {{KID_ATTN_W64, KID_ATTN_DQ_W64, KID_ATTN_DK_W64, KID_ATTN_DV_W64, KID_NONE}, {KID_ATTNB_W64, KID_ATTNB_DQ_W64, KID_ATTNB_DK_W64, KID_ATTNB_DV_W64, KID_ATTNB_DB_W64}};
    const int through_lds[2][5] = {{KID_ATTN_T64, KID_ATTN_DQ_T64, KID_ATTN_DK_T64, KID_ATTN_DV_T64, KID_NONE}, {KID_ATTNB_T64, KID_ATTNB_DQ_T64, KID_ATTNB_DK_T64, KID_ATTNB_DV_T64, KID_ATTNB_DB_T64}};
    p.kid = waves[biased][of_op] + (narrow ? 0 : 1);
    const long columns = by_keys ? Tk : group * Tq;
    long per_block = 16, other = 64, few = 4;                  // columns of a workgroup, the other side's in a block, blocks a split has at least
    // Straight from memory with 16 columns a wavefront, or 128 columns a workgroup through LDS. The former where there are few
    // columns, and where the whole task is a wavefront and block for each of at most 768 wavefronts, three on a compute unit, which
    // then takes as long as one block. Forward, us straight / through LDS: 256 x 256 with one head 7.0 / 13.4 (64 wavefronts), 128 x 77
    // with 16 heads 7.4 / 9.4 (256), 48 x 512 with 32 heads of 128 17.5 / 23.4 (768), 64 x 64 with 256 heads 13.1 / 6.5 (1024), 256 x 77 with
    // 64 heads 17.5 / 8.9 (2048); dq 12.4 / 13.3, 11.8 / 13.6, 24.4 / 29.5, 23.5 / 12.3, 19.6 / 12.6. dk and dv share a launch through LDS with up
    // to 64 channels; with more, 128 x 128 with four heads 21 + 15 / 24 + 18 (64), 48 x 512 with 32 heads 49 + 35 / 18 + 13 (1024).
    const long wavefronts = q.n * nd.p.kv_heads * ceil_div(columns, 16) * (by_keys ? group * ceil_div(Tq, 64) : ceil_div(Tk, 64));
    // With a bias the tile kernels' columns are of one head, which has to have enough of them.
    const bool by_heads = biased && !by_keys;
    const bool tiles = !g->unsplit_products && (by_heads ? Tq : columns) > 32 && (wavefronts > 768 || (by_keys && narrow));
    if (tiles) {
        p.kid = through_lds[biased][of_op] + (narrow ? 0 : 1);
        per_block = kAttentionColumns, few = 1;
        other = nd.op != NG_OP_ATTENTION ? kGradientBlock : narrow ? attention_block<64>() : attention_block<128>();
    }
    p.query_blocks = (int)ceil_div(Tq, per_block);
    p.col_blocks = (int)(by_heads && (tiles || dbias) ? group * p.query_blocks : ceil_div(columns, per_block));
    const long groups = q.n * nd.p.kv_heads * p.col_blocks, blocks = by_keys ? group * ceil_div(Tq, other) : ceil_div(Tk, other);
    long want = 1;
    if (per_block == kAttentionColumns)
        want = tile_splits(nd.op, narrow, groups, blocks);
    else                                                       // up to 1024 workgroups
        want = std::max<long>(1, std::min<long>({ceil_div(blocks, few), ceil_div(1024, groups), kMaxWaveSplits, std::lround(std::sqrt(6.0 * (double)blocks))}));
    want = knob_int("NG_ATTN_SPLITS", 1, 32, want);
    p.per_split = (int)(ceil_div(ceil_div(blocks, want), few) * few);
    p.splits = (int)ceil_div(blocks, p.per_split);
    p.tiles = groups * p.splits;
    if (dbias) {                                               // for each head: rows of sums of its workgroups, and of groups of them
        const long rows = q.n * p.query_blocks * p.splits, sums = row_groups((int)rows), distances = g->nodes[nd.preds.back()].out.h * g->nodes[nd.preds.back()].out.w;
        p.ws_floats = (size_t)round64(nd.p.heads * (rows + sums) * ((distances + 3) & ~3L));
        p.cnt_words = (size_t)round64(nd.p.heads * (1 + sums));
    } else if (p.splits > 1) {
        p.ws_floats = (size_t)round64(p.tiles * (d + (nd.op == NG_OP_ATTENTION ? 2 : 0)) * per_block);
        p.cnt_words = (size_t)round64(groups);
    }
    if (nd.op == NG_OP_ATTENTION)
        for (const Node& r : g->nodes)
            if (r.op == NG_OP_ATTENTION_ROWS && r.preds[1] == v) p.stats_floats = (size_t)round64(2 * q.n * nd.p.heads * Tq);
    return p;
}
struct RopePlan {
    int kid = KID_NONE;
    int blocks = 0, heads_per_tile = 1, items = 1, per_tile = 1;
    long tiles = 0;
    size_t ws_floats = 0, cnt_words = 0;
};
bool is_rope_op(int op) { return op >= NG_OP_HEAD_ROPE && op <= NG_OP_HEAD_ROPE_WGRAD; }
RopePlan rope_plan(const ng_graph* g, int v) {
    RopePlan p;
    const Node& nd = g->nodes[v];
    if (!is_rope_op(nd.op)) return p;
    const int which = nd.op - NG_OP_HEAD_ROPE;                 // forward, dgrad, wgrad: in the order of the kernel ids
    const Shape& x = g->nodes[nd.preds[which ? 1 : 0]].out;
    const long d = x.c / nd.p.heads, T = x.h * x.w, H = nd.p.heads;
    const bool wgrad = nd.op == NG_OP_HEAD_ROPE_WGRAD;
    // workgroups: enough to fill the GPU; every one of wgrad's leaves a row of sums that somebody has to add up
    const long most = wgrad ? 512 : 1L << 20;
    if (T < 16) {
        p.kid = KID_ROPE_N + 3 * which;
        const long groups = ceil_div(x.n * H * T, 4);
        p.per_tile = (int)ceil_div(groups, most);
        p.tiles = ceil_div(groups, p.per_tile);
    } else {
        p.kid = (d <= 128 ? KID_ROPE_4 : KID_ROPE_8) + 3 * which;
        p.blocks = (int)ceil_div(T, 64);
        p.items = (int)(x.n * p.blocks);
        // (wgrad, and with it both gradients in one launch, has two workgroups on a compute unit: 700 blocks of heads of 64 channels by
        // themselves take two turns and 22 us, two of a workgroup 17)
        p.heads_per_tile = (int)std::max<long>(1, std::min<long>(H, wgrad ? ceil_div((long)p.items * H, 512) : (long)p.items * H / 1024));
        p.per_tile = (int)ceil_div(p.items, most);
        p.tiles = ceil_div(p.items, p.per_tile) * ceil_div(H, p.heads_per_tile);
    }
    if (wgrad) {
        p.ws_floats = (size_t)round64(p.tiles * d);
        p.cnt_words = (size_t)round64(1 + ceil_div(p.tiles, kGammaGroup));
    }
    return p;
}
// How a layer norm is computed: threads side by side along the tokens (wider accesses in a row, fewer channels in registers), and how
// many blocks of tokens a workgroup walks.
struct NormPlan {
    int kid = KID_NONE;
    int lanes_log2 = 0, blocks = 1, items = 1, per_tile = 1;
    long tiles = 0;
    size_t ws_floats = 0, cnt_words = 0;
};
bool is_norm_op(int op) { return op >= NG_OP_LAYER_NORM && op <= NG_OP_LAYER_NORM_WGRAD; }
NormPlan norm_plan(const ng_graph* g, int v) {
    NormPlan p;
    const Node& nd = g->nodes[v];
    if (!is_norm_op(nd.op)) return p;
    const int which = nd.op - NG_OP_LAYER_NORM;                // forward, dgrad, wgrad
    const Shape& x = g->nodes[nd.preds[which ? 1 : 0]].out;
    const long C = x.c, T = x.h * x.w;
    const bool wgrad = nd.op == NG_OP_LAYER_NORM_WGRAD;
    long most = 512;                                           // workgroups of wgrad
    auto one_of = [which](int forward, int dgrad, int wgrad) { return which == 0 ? forward : which == 1 ? dgrad : wgrad; };
    if (T < 4)
        while ((1L << p.lanes_log2) < T) ++p.lanes_log2;
    // (What no workgroup holds in registers is read again for each sum, much slower: 2 images of 5120 channels, 2048 tokens, with gradients, in 1024
    // threads of 16 channels each 202 us, read again 972; 8192 channels, 8192 tokens 666 and 2079.)
    if (C > norm_channels(T < 4 ? KID_NORM_S16 : KID_NORM_W16, T < 4 ? p.lanes_log2 : 0)) {
        p.kid = one_of(KID_NORM_M, KID_NORM_DX_M, KID_NORM_DG_M);
        while (p.lanes_log2 < 4 && (1L << p.lanes_log2) < T) ++p.lanes_log2;
        p.blocks = (int)ceil_div(T, 1L << p.lanes_log2);
    } else if (T < 4) {
        p.kid = one_of(KID_NORM_S16, KID_NORM_DX_S16, KID_NORM_DG_S16);
    } else {
        // Threads side by side along the tokens, 1, 2, 4 or 8 with four tokens each: as many as the rules below allow, because what a workgroup
        // reads of a channel should be whole lines of memory. (Images x channels x tokens; both: the gradients in one launch.)
        //   TB/s with 2 / 4 / 8: forward of 16 x 512 x 8192 3.3 / 4.1 / 5.1, of 16 x 1024 x 4096 2.9 / 3.9 / 4.8; both 3.3 / 3.7 / 4.3 and 2.8 / 3.5 / 3.9.
        // Rule 1: at least 64 workgroups, 128 of more than 256 threads, 256 of more than 512; few of them have few rows of sums to join.
        //   us with 64 / 128 / 256 at least: forward and both of 4 x 256 x 400 15.4 / 16.8 / 19.5, of 6 x 520 x 333, where 64 are of 1024 threads,
        //   27.0 / 21.6 / 24.9. Both of 16 x 1000 x 300 in 160 workgroups of 1024 threads 29.3, in twice as many of 512 26.2.
        // Rule 2: eight with more than 256 threads only for tensors beyond the 256 MB cache behind the L2s.
        //   us with 4 / 8: forward of 4 x 2048 x 4096 (in the cache) 44 / 51, both of 8 x 1024 x 2048 (in it) 49 / 58, of 8 x 1024 x 4096 121 / 115.
        // Rule 3: more channels than 512 threads of 8 hold: forward in 512 threads of 16 channels each, not 1024 of 8.
        //   us with 1024 / 512: 16 x 1024 x 4096 123 / 113, 8 x 1024 x 4096 (in the cache) 53 / 39, eight side by side.
        // Rule 4: more than 1024 threads of 8 hold: 16 each. The gradients then read dy twice, with twice as many tokens side by side.
        //   us of both with 8 / 16 channels a thread: 2 x 4096 x 8192 397 / 313, 2 x 4096 x 2000 71 / 67, 8 x 2048 x 4096 262 / 225.
        const bool large = (double)x.elems() * 4 * (which == 0 ? 2 : 3) > 268435456.0;
        long threads = 0;
        for (int log2 = 3; log2 >= 0; --log2) {
            const long lanes = 1L << log2;
            threads = ceil_div(C * lanes, 8);
            if (log2 > 0 && (2 * lanes >= T || threads > 2048 || x.n * ceil_div(T, 4 * lanes) < (threads <= kBlock ? 64 : threads <= 512 ? 128 : 256))) continue;
            if (log2 == 3 && threads > kBlock && !large) continue;
            p.lanes_log2 = log2;
            break;
        }
        p.kid = threads <= kBlock ? one_of(KID_NORM_V8, KID_NORM_DX_V8, KID_NORM_DG_V8)
              : which == 0 && p.lanes_log2 == 0 && threads <= 512 ? (int)KID_NORM_V16            // few tokens: a kernel that the device-resident replay has as well
              : threads <= 512 ? one_of(KID_NORM_H8, KID_NORM_DX_H8, KID_NORM_DG_H8)
              : threads <= 1024 ? one_of(KID_NORM_H16, KID_NORM_DX_W8, KID_NORM_DG_W8) : one_of(KID_NORM_W16, KID_NORM_DX_W16, KID_NORM_DG_W16);      // (16 channels a thread)
        p.blocks = (int)ceil_div(T, 4L << p.lanes_log2);
        if (p.kid != KID_NORM_DG_V8) most = 256;                // one workgroup of so many threads and registers on a compute unit, all of them at once
    }
    p.items = (int)(x.n * p.blocks);
    p.per_tile = (int)ceil_div(p.items, wgrad ? most : 1L << 20);      // every workgroup of wgrad's leaves a row of sums that somebody has to add up
    p.tiles = ceil_div(p.items, p.per_tile);
    if (wgrad) {
        p.ws_floats = (size_t)round64((p.tiles + row_groups((int)p.tiles)) * ((2 * C + 3) & ~3L));
        p.cnt_words = (size_t)round64(1 + row_groups((int)p.tiles));
    }
    return p;
}
// Bucket of each distance -max_distance .. max_distance, -1 for keys that are not seen.
std::vector<int> position_buckets(const ng_op_params& p) {
    const int m = p.max_distance, b = p.both ? p.buckets / 2 : p.buckets, exact = b / 2;
    std::vector<int> of(2 * (size_t)m + 1);
    for (int d = -m; d <= m; ++d) {
        const int far = d < 0 ? -d : d;
        int at = far;
        if (far >= exact) {
            const double steps = std::log((double)far / exact) / std::log((double)m / exact) * (b - exact);
            at = std::min(b - 1, exact + (int)std::floor(steps + 1e-9));
        }
        of[(size_t)(d + m)] = d > 0 ? (p.both ? b + at : -1) : at;
    }
    return of;
}
bool is_position_bias_op(int op) { return op == NG_OP_POSITION_BIAS || op == NG_OP_POSITION_BIAS_WGRAD; }
}  // namespace

size_t packed_floats(const ng_graph* g, int v) {
    const Node& nd = g->nodes[v];
    if (is_norm_op(nd.op)) {
        const NormPlan p = norm_plan(g, v);
        return p.ws_floats + p.cnt_words;
    }
    if (is_position_bias_op(nd.op)) return 2 * (size_t)nd.p.max_distance + 1;      // the buckets
    if (is_attention_op(nd.op)) {
        const AttentionPlan p = attention_plan(g, v);
        return p.ws_floats + p.cnt_words + p.stats_floats;
    }
    if (is_rope_op(nd.op)) {
        const RopePlan p = rope_plan(g, v);
        return p.ws_floats + p.cnt_words;
    }
    long wm, wn, wk;
    if (wgrad_dims(g, v, &wm, &wn, &wk)) {                     // split-K workspace: partial tiles, then the arrival counters
        const WgradPlan p = wgrad_plan(g, v);
        return p.ws_floats + p.cnt_words;
    }
    if (nd.op == NG_OP_DWCONV_WGRAD) {                         // per-chunk partial sums [C][chunks][K K] (padded), then one arrival counter per channel
        const Shape& x = g->nodes[nd.preds[1]].out;
        const long chunks = dw_wgrad_chunks(x.c, x.n);
        return chunks > 1 ? (size_t)((x.c * chunks * nd.p.k * nd.p.k + 63) & ~63L) + (size_t)((x.c + 63) & ~63L) : 0;
    }
    if (nd.op == NG_OP_BN_ACT_WGRAD) {                         // per-chunk sums [C][chunks][2] (padded), then one arrival counter per channel
        const Shape& x = g->nodes[nd.preds[1]].out;
        const long chunks = bn_wgrad_chunks(x.c, x.n);
        return chunks > 1 ? (size_t)((x.c * chunks * 2 + 63) & ~63L) + (size_t)((x.c + 63) & ~63L) : 0;
    }
    if (g->trainable) return 0;                                // weights change between replays: nothing is folded or repacked
    if (nd.op == NG_OP_BN_ACT) return 2 * (size_t)((nd.out.c + 3) & ~3L);   // folded scale, shift
    if (nd.op == NG_OP_CONV3X3) return choose_c3(g, v).packed;
    return choose_pw(g, v).packed;
}

bool has_arrival_counters(int op) {
    return op == NG_OP_CONV1X1_WGRAD || op == NG_OP_CONV3X3_WGRAD || op == NG_OP_DWCONV_WGRAD || op == NG_OP_BN_ACT_WGRAD || is_attention_op(op) || is_rope_op(op) || is_norm_op(op);
}

namespace {
__global__ __launch_bounds__(kBlock) void clear_words_kernel(float* p, size_t words) {
    for (size_t i = (size_t)blockIdx.x * kBlock + threadIdx.x; i < words; i += (size_t)gridDim.x * kBlock) p[i] = 0.f;
}
// (a kernel: ng_replay_static, which records no memset, may have to do it)
hipError_t clear_words(float* p, size_t words, void* stream) {
    clear_words_kernel<<<dim3((unsigned)std::min<size_t>((words + kBlock - 1) / kBlock, 1024)), dim3(kBlock), 0, static_cast<hipStream_t>(stream)>>>(p, words);
    return hipGetLastError();
}
}  // namespace

// Fill node v's constant memory: one pass over the weights, at bind time.
int pack_constants(ng_graph* g, int v, float* packed, void* stream) {
    const Node& nd = g->nodes[v];
    long wm, wn, wk;
    if (is_attention_op(nd.op) || is_rope_op(nd.op) || is_norm_op(nd.op)) {    // the arrival counters start at zero
        const AttentionPlan p = attention_plan(g, v);
        const RopePlan r = rope_plan(g, v);
        const NormPlan m = norm_plan(g, v);
        const size_t words = p.cnt_words + r.cnt_words + m.cnt_words;
        if (words == 0) return NG_OK;
        const hipError_t e = clear_words(packed + p.ws_floats + r.ws_floats + m.ws_floats, words, stream);
        if (e != hipSuccess) return g->fail(NG_EHIP, "clearing arrival counters of an attention operator or a norm: %s", hipGetErrorString(e));
        return NG_OK;
    }
    if (is_position_bias_op(nd.op)) {
        const std::vector<int> of = position_buckets(nd.p);
        hipError_t e = hipMemcpyAsync(packed, of.data(), of.size() * sizeof(int), hipMemcpyHostToDevice, static_cast<hipStream_t>(stream));
        if (e == hipSuccess) e = hipStreamSynchronize(static_cast<hipStream_t>(stream));      // (the host's copy ends here)
        if (e != hipSuccess) return g->fail(NG_EHIP, "copying the buckets of a position bias: %s", hipGetErrorString(e));
        return NG_OK;
    }
    if (nd.op == NG_OP_DROPOUT) return NG_OK;
    if (wgrad_dims(g, v, &wm, &wn, &wk)) {                     // the arrival counters start at zero
        const WgradPlan p = wgrad_plan(g, v);
        if (p.cnt_words == 0) return NG_OK;
        const hipError_t e = clear_words(packed + p.ws_floats, p.cnt_words, stream);
        if (e != hipSuccess) return g->fail(NG_EHIP, "clearing split-K counters: %s", hipGetErrorString(e));
        return NG_OK;
    }
    if (nd.op == NG_OP_DWCONV_WGRAD || nd.op == NG_OP_BN_ACT_WGRAD) {
        const size_t floats = packed_floats(g, v);
        if (floats == 0) return NG_OK;
        const size_t cnt = (size_t)((g->nodes[nd.preds[1]].out.c + 63) & ~63L);
        const hipError_t e = clear_words(packed + floats - cnt, cnt, stream);
        if (e != hipSuccess) return g->fail(NG_EHIP, "clearing depthwise wgrad counters: %s", hipGetErrorString(e));
        return NG_OK;
    }
    if (g->trainable) return NG_OK;
    if (nd.op == NG_OP_BN_ACT) {
        for (int j = 0; j < 4; ++j)
            if (!nd.weights[j]) return g->fail(NG_EINVAL, "node %d: weight %d is a null device pointer", v, j);
        const int C = (int)nd.out.c;
        fold_bn_kernel<<<dim3((unsigned)((C + kBlock - 1) / kBlock)), dim3(kBlock), 0, static_cast<hipStream_t>(stream)>>>(
            static_cast<const float*>(nd.weights[0]), static_cast<const float*>(nd.weights[1]),
            static_cast<const float*>(nd.weights[2]), static_cast<const float*>(nd.weights[3]), nd.p.eps, packed,
            packed + ((C + 3) & ~3), C);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return g->fail(NG_EHIP, "folding batch-norm parameters: %s", hipGetErrorString(e));
        return NG_OK;
    }
    const bool c3 = nd.op == NG_OP_CONV3X3;
    const PwChoice c = c3 ? choose_c3(g, v) : choose_pw(g, v);
    if (c.packed == 0) return NG_OK;
    const int cin = (int)g->nodes[nd.preds[0]].out.c * (c3 ? 9 : 1), cout = (int)nd.out.c;
    if (!nd.weights[0]) return g->fail(NG_EINVAL, "node %d: weight 0 is a null device pointer", v);
    const dim3 grid((unsigned)((c.packed + kBlock - 1) / kBlock)), block(kBlock);
    if (c.kind == PwChoice::PW_PATCH || c.kind == PwChoice::C3_PATCH) {
        const long threads = (long)(c.packed / 12);             // one per 8 weights in three parts of 16 bits
        pack_split_weights_kernel<<<dim3((unsigned)ceil_div(threads, kBlock)), block, 0, static_cast<hipStream_t>(stream)>>>(
            static_cast<const float*>(nd.weights[0]), packed, cout, c.groups, c3 ? 9 : 1,
            (int)(c.packed / ((size_t)cin / 16 * (kSplitFragBytes / 4))), threads);
    }
    else if (c.kind == PwChoice::LDS64)
        pack_pw_lds_weights_kernel<<<grid, block, 0, static_cast<hipStream_t>(stream)>>>(
            static_cast<const float*>(nd.weights[0]), packed, cout, cin, (int)(c.packed / (size_t)c.groups), (long)c.packed);
    else if (c.kind == PwChoice::C3_LDS)
        pack_c3_lds_weights_kernel<<<grid, block, 0, static_cast<hipStream_t>(stream)>>>(
            static_cast<const float*>(nd.weights[0]), packed, cout, cin / 9, c.groups, (int)(c.packed / (9 * (size_t)c.groups)), (long)c.packed);
    else if (c.kind == PwChoice::DIRECT32)
        pack_pw_weights_kernel<<<grid, block, 0, static_cast<hipStream_t>(stream)>>>(
            static_cast<const float*>(nd.weights[0]), packed, cout, cin, c.groups, (int)c.packed);
    else
        pack_pw_weights_k4_kernel<<<grid, block, 0, static_cast<hipStream_t>(stream)>>>(
            static_cast<const float*>(nd.weights[0]), packed, cout, cin, c.groups, (int)c.packed);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return g->fail(NG_EHIP, "repacking conv1x1 weights: %s", hipGetErrorString(e));
    return NG_OK;
}

// set_kernel for a kernel that a plan has chosen among those that take the same arguments
template <class A>
static void set_any_kernel(Task& t, int kid, const A& a, long ntiles) {
    switch (kid) {
#define NG_CASE(KID)                                                                             \
    case KID:                                                                                    \
        if constexpr (std::is_same<typename KernelOf<KID>::Args, A>::value) set_kernel<KID>(t, a, ntiles); \
        break;
        NG_FOR_EACH_KID(NG_CASE)
#undef NG_CASE
        default: break;
    }
}

int build_task(ng_graph* g, int v, char* arena, float* packed, Task& t) {
    const Node& nd = g->nodes[v];
    t = Task();
    t.block[0] = kBlock;
    if (nd.op == NG_OP_INPUT) return NG_OK;
    for (size_t j = 0; j < nd.weights.size(); ++j)
        if (!nd.weights[j] && !g->dry_run) return g->fail(NG_EINVAL, "node %d: weight %d is a null device pointer", v, (int)j);

    auto buf = [&](int id) { return reinterpret_cast<float*>(arena + g->offset[id]); };
    const Shape& o = nd.out;
    const Shape& i0 = nd.preds.empty() ? o : g->nodes[nd.preds[0]].out;
    const int total = (int)o.elems();
    const int hw_out = (int)(o.h * o.w);
    auto wf = [&](int j) { return static_cast<const float*>(nd.weights[j]); };

    switch (nd.op) {
        case NG_OP_BN_ACT:
            if (g->trainable) {                                   // gamma and beta change between replays: no folded copy
                BnRawArgs a{};
                a.x = buf(nd.preds[0]), a.y = buf(v);
                a.gamma = wf(0), a.beta = wf(1), a.mean = wf(2), a.var = wf(3);
                a.eps = nd.p.eps, a.relu = nd.p.relu != 0;
                a.C = (int)o.c, a.HW = hw_out, a.N = (int)o.n, a.total = total;
                set_kernel<KID_BN_RAW>(t, a, ceil_div(total, kBlock));
                break;
            }
            [[fallthrough]];
        case NG_OP_RELU: {
            BnArgs a{};
            a.x = buf(nd.preds[0]);
            a.y = buf(v);
            if (nd.op == NG_OP_BN_ACT) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for folded batch-norm parameters", v);
                a.scale = packed, a.shift = packed + ((o.c + 3) & ~3L);
                a.relu = nd.p.relu != 0;
            } else {
                a.relu = 1;
            }
            a.C = (int)o.c, a.HW = hw_out, a.total = total;
            a.cols = (int)(o.n * hw_out);
            if (hw_out % 4 == 0) set_kernel<KID_BN_V4>(t, a, ceil_div(total / 4, kBlock));
            else set_kernel<KID_BN>(t, a, ceil_div(total, kBlock));
            break;
        }
        case NG_OP_ADD_N: {
            AddArgs a{};
            a.k = (int)nd.preds.size();
            for (int j = 0; j < NG_MAX_PREDS; ++j) a.x[j] = buf(nd.preds[j < a.k ? j : 0]);
            a.y = buf(v);
            a.total = total;
            a.C = (int)o.c, a.HW = hw_out, a.cols = (int)(o.n * hw_out);
            if (total % 4 == 0) set_kernel<KID_ADD_V4>(t, a, ceil_div(total / 4, kBlock));
            else set_kernel<KID_ADD>(t, a, ceil_div(total, kBlock));
            break;
        }
        case NG_OP_CONCAT: {
            ConcatArgs a{};
            a.k = (int)nd.preds.size();
            int first = 0;
            for (int j = 0; j < a.k; ++j) {
                a.x[j] = buf(nd.preds[j]);
                a.cin[j] = (int)g->nodes[nd.preds[j]].out.c;
                a.lo[j] = nd.p.slice_lo[j];
                a.first[j] = first;
                first += nd.p.slice_hi[j] - nd.p.slice_lo[j];
            }
            for (int j = a.k; j < NG_MAX_PREDS; ++j) a.x[j] = a.x[0], a.first[j] = first;
            a.y = buf(v);
            a.C = (int)o.c, a.HW = hw_out, a.total = total;
            // 128 bits at a time wherever four elements never straddle two blocks or two images, on either side: every block
            // starts at and has a multiple of four elements (odd maps with channels in fours as well; an Inception-style
            // network at batch 32, whose concats are of 35 x 35 and 17 x 17 maps, 3666 -> 3571 us)
            bool quads = true;
            for (int j = 0; j < a.k; ++j)
                quads = quads && (long)a.first[j] * hw_out % 4 == 0 && (long)a.lo[j] * hw_out % 4 == 0 && (long)a.cin[j] * hw_out % 4 == 0;
            quads = quads && (long)a.C * hw_out % 4 == 0;
            if (quads) set_kernel<KID_CONCAT_V4>(t, a, ceil_div(total / 4, kBlock));
            else set_kernel<KID_CONCAT>(t, a, ceil_div(total, kBlock));
            break;
        }
        case NG_OP_POOL: {
            PoolArgs a{buf(nd.preds[0]), buf(v), (int)i0.h, (int)i0.w, (int)o.h, (int)o.w,
                       nd.p.stride, nd.p.pad, nd.p.pool_mode, total};
            // large tensors (batches): four outputs of a column per thread
            if (total >= kPoolRowMinOutputs && (nd.p.stride == 1 || nd.p.stride == 2)) {
                const long items = (long)o.n * o.c * ceil_div(o.h, 4) * o.w;
                if (nd.p.stride == 1) set_kernel<KID_POOL_ROW_S1>(t, a, ceil_div(items, kBlock));
                else set_kernel<KID_POOL_ROW_S2>(t, a, ceil_div(items, kBlock));
                break;
            }
            set_kernel<KID_POOL>(t, a, ceil_div(total, kBlock));
            break;
        }
        case NG_OP_DWCONV: {
            DwArgs a{buf(nd.preds[0]), wf(0), buf(v), (int)o.c, (int)i0.h, (int)i0.w, (int)o.h, (int)o.w, total};
            const long n = ceil_div(total, kBlock);
            // large tensors of small planes (batches): whole planes through LDS, four outputs per thread
            const long quads = i0.h * ceil_div(i0.w, 4), per_wg = planes_in_lds((int)i0.h, (int)i0.w, nd.p.k);
            if (total >= kDwLdsMinOutputs && (nd.p.k == 3 || nd.p.k == 5) && (nd.p.stride == 1 || nd.p.stride == 2) && i0.w >= 4 &&
                o.w >= 4 && per_wg > 0 && o.h * ceil_div(o.w, 4) <= quads) {
                a.K = nd.p.k, a.S = nd.p.stride, a.planes_per_tile = (int)per_wg;
                set_kernel<KID_DW_LDS>(t, a, ceil_div((long)o.n * o.c, per_wg));
                break;
            }
            if (nd.p.k == 3 && nd.p.stride == 1) set_kernel<KID_DW_K3S1>(t, a, n);
            else if (nd.p.k == 3) set_kernel<KID_DW_K3S2>(t, a, n);
            else if (nd.p.stride == 1) set_kernel<KID_DW_K5S1>(t, a, n);
            else set_kernel<KID_DW_K5S2>(t, a, n);
            break;
        }
        case NG_OP_GLOBAL_AVGPOOL: {
            GapArgs a{buf(nd.preds[0]), buf(v), (int)(i0.h * i0.w), (int)(o.n * o.c)};
            set_kernel<KID_GAP>(t, a, ceil_div(a.planes, kBlock / 64));
            break;
        }
        case NG_OP_FC:
        case NG_OP_CONV1X1: {
            const bool fc = nd.op == NG_OP_FC;
            if (g->trainable) {                                   // weights change between replays: read them where they are
                GemmArgs a{};
                a.a = wf(0), a.b = buf(nd.preds[0]), a.c = buf(v), a.bias = fc ? wf(1) : nullptr;
                a.M = (int)o.c, a.K = (int)i0.c, a.N = (int)(o.n * hw_out);
                a.Cin = (int)i0.c, a.Cout = (int)o.c, a.H = a.Ho = (int)o.h, a.W = a.Wo = (int)o.w, a.stride = 1;
                a.tiles_n = (int)ceil_div(a.N, kGemmTile), a.splits = 1, a.k_per_split = a.K;
                if (hw_out == 1 && (long)a.M * a.N <= kSmallGemmOutputs && a.K <= kSmallGemmK) {
                    // Y[n][o] = sum_k W[o][k] X[n][k] + b[o]
                    SmallGemmArgs sg{a.a, a.b, a.c, a.bias, a.M, a.N, a.K, a.K, 1, 1, a.K, 1, a.M, 0};
                    set_small_gemm(t, sg, [](Task& tt, const SmallGemmArgs& aa, long n) { set_kernel<KID_SMALL_GEMM>(tt, aa, n); });
                    break;
                }
                if (!fc && pw_px_applies(a)) set_kernel<KID_PW_PX_FWD>(t, a, pw_px_tiles(a));
                else set_kernel<KID_GEMM_PW_FWD>(t, a, (long)a.tiles_n * ceil_div(a.M, kGemmTile));
                break;
            }
            const PwChoice c = choose_pw(g, v);
            if (c.kind == PwChoice::GEMV) {
                FcArgs a{buf(nd.preds[0]), wf(0), wf(1), buf(v), (int)o.n, (int)i0.c, (int)o.c};
                set_kernel<KID_FC_GEMV>(t, a, ceil_div(a.Cout, kBlock / 64));
                break;
            }
            PwArgs a{};
            a.x = buf(nd.preds[0]), a.w = wf(0), a.bias = fc ? wf(1) : nullptr, a.y = buf(v);
            a.Cin = (int)i0.c, a.Cout = (int)o.c, a.HW = hw_out, a.cols = (int)(o.n * hw_out);
            if (c.kind == PwChoice::PW_PATCH) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for repacked weights", v);
                a.wp = packed, a.ksteps = c.groups;
                a.tiles_n = (int)ceil_div(a.cols, 64);
                a.mtiles = (int)ceil_div(a.Cout, c.kid == KID_PW_P32 ? 32 : 64);
                if (c.kid == KID_PW_P32) set_kernel<KID_PW_P32>(t, a, (long)a.tiles_n * a.mtiles);
                else set_kernel<KID_PW_P64>(t, a, (long)a.tiles_n * a.mtiles);
                break;
            }
            if (c.kind == PwChoice::LDS64) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for repacked weights", v);
                a.wp = packed, a.ksteps = c.groups;
                a.tiles_n = (int)ceil_div(a.cols, 64);
                set_kernel<KID_PW_64>(t, a, (long)a.tiles_n * ceil_div(a.Cout, 64));
                break;
            }
            if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for repacked weights", v);
            a.wp = packed;
            a.ksteps = c.groups;
            a.mtiles = (int)ceil_div(a.Cout, 16);
            if (c.kind == PwChoice::DIRECT32) {
                a.tiles_n = (int)ceil_div(a.cols, 32);
                const long n = (long)a.tiles_n * ceil_div(a.Cout, 32);
                if (c.in_flight == 4) set_kernel<KID_PW_D4>(t, a, n);
                else if (c.in_flight == 8) set_kernel<KID_PW_D8>(t, a, n);
                else set_kernel<KID_PW_D16>(t, a, n);
            } else if (c.kind == PwChoice::K4_VEC) {
                a.tiles_n = (int)ceil_div(a.cols, 64);
                const long n = (long)a.tiles_n * a.mtiles;
                if (c.in_flight == 1) set_kernel<KID_PW_V1>(t, a, n);
                else if (c.in_flight == 2) set_kernel<KID_PW_V2>(t, a, n);
                else if (c.in_flight == 3) set_kernel<KID_PW_V3>(t, a, n);
                else set_kernel<KID_PW_V4>(t, a, n);
            } else {
                a.tiles_n = (int)ceil_div(a.cols, 16);
                const long n = (long)a.tiles_n * a.mtiles;
                if (c.in_flight == 1) set_kernel<KID_PW_S1>(t, a, n);
                else if (c.in_flight == 2) set_kernel<KID_PW_S2>(t, a, n);
                else if (c.in_flight == 3) set_kernel<KID_PW_S3>(t, a, n);
                else set_kernel<KID_PW_S4>(t, a, n);
            }
            break;
        }
        case NG_OP_CONV3X3: {
            C3Args a{};
            a.x = buf(nd.preds[0]), a.w = wf(0), a.y = buf(v);
            a.Cin = (int)i0.c, a.Cout = (int)o.c, a.H = (int)i0.h, a.W = (int)i0.w, a.Ho = (int)o.h, a.Wo = (int)o.w;
            a.pad = nd.p.pad, a.stride = nd.p.stride;
            if (g->trainable) {
                GemmArgs ga{};
                ga.a = wf(0), ga.b = buf(nd.preds[0]), ga.c = buf(v);
                ga.M = (int)o.c, ga.K = (int)i0.c * 9, ga.N = (int)(o.n * o.h * o.w);
                ga.Cin = (int)i0.c, ga.Cout = (int)o.c, ga.H = (int)i0.h, ga.W = (int)i0.w, ga.Ho = (int)o.h, ga.Wo = (int)o.w;
                ga.stride = nd.p.stride, ga.pad = nd.p.pad;
                ga.tiles_n = (int)ceil_div(ga.N, kGemmTile), ga.splits = 1, ga.k_per_split = ga.K;
                set_kernel<KID_GEMM_C3_FWD>(t, ga, (long)ga.tiles_n * ceil_div(ga.M, kGemmTile));
                break;
            }
            const PwChoice c = choose_c3(g, v);
            if (c.kind == PwChoice::C3_PATCH) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for repacked weights", v);
                a.wp = packed, a.groups = c.groups;
                a.cols = (int)(o.n * o.h * o.w);
                for (const PatchKernel& k : kPatchKernels) {
                    if (k.kid != c.kid) continue;
                    // runs of pixels per image; conv3x3_mfma_split_k takes rows of whole width
                    const Strips strips = k.kid == KID_C3_SK ? Strips{o.w, ceil_div(o.h * o.w, k.tn)} : choose_strips(k.kid, k.tn, o.h, o.w, nd.p.stride);
                    a.tiles_x = (int)strips.width, a.tiles_xy = (int)strips.runs;
                    a.tiles_n = (int)o.n * a.tiles_xy;
                    a.co_groups = (int)ceil_div(a.Cout, k.tm);
                }
                const long n = (long)a.tiles_n * a.co_groups;
                switch (c.kid) {
                    case KID_C3_P64: set_kernel<KID_C3_P64>(t, a, n); break;
                    case KID_C3_P96: set_kernel<KID_C3_P96>(t, a, n); break;
                    case KID_C3_Q32: set_kernel<KID_C3_Q32>(t, a, n); break;
                    case KID_C3_Q64: set_kernel<KID_C3_Q64>(t, a, n); break;
                    case KID_C3_R32: set_kernel<KID_C3_R32>(t, a, n); break;
                    case KID_C3_R128: set_kernel<KID_C3_R128>(t, a, n); break;
                    case KID_C3_SK: set_kernel<KID_C3_SK>(t, a, n); break;
                    default: set_kernel<KID_C3_Q128>(t, a, n); break;
                }
                break;
            }
            if (c.kind == PwChoice::C3_LDS) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for repacked weights", v);
                a.wp = packed, a.groups = c.groups;
                a.cols = (int)(o.n * o.h * o.w);
                if (a.Cout <= 32) {
                    a.tiles_n = (int)ceil_div(a.cols, 128);
                    set_kernel<KID_C3_L32>(t, a, (long)a.tiles_n * ceil_div(a.Cout, 32));
                } else {
                    a.tiles_n = (int)ceil_div(a.cols, 64);
                    set_kernel<KID_C3_L64>(t, a, (long)a.tiles_n * ceil_div(a.Cout, 64));
                }
                break;
            }
            if (c.packed != 0) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for repacked weights", v);
                a.wp = packed, a.groups = c.groups;
                a.cols = (int)(o.n * o.h * o.w), a.tiles_n = (int)ceil_div(a.cols, 16);
                const long n = (long)a.tiles_n * ceil_div(a.Cout, 16);
                if (c.in_flight == 1) set_kernel<KID_C3_M1>(t, a, n);
                else if (c.in_flight == 2) set_kernel<KID_C3_M2>(t, a, n);
                else if (c.in_flight == 3) set_kernel<KID_C3_M3>(t, a, n);
                else set_kernel<KID_C3_M4>(t, a, n);
                break;
            }
            // small maps: 8 x 8 tiles waste fewer lanes; a stem at batch 1 (3 input channels, a large map): four times the
            // workgroups, each with a quarter of the patch to load
            const bool small = o.h * o.w <= 24 * 24 || (a.Cin <= 4 && o.n == 1);
            const int tp = small ? 8 : 16;
            a.tiles_x = (int)ceil_div(o.w, tp);
            a.tiles_xy = a.tiles_x * (int)ceil_div(o.h, tp);
            a.co_groups = (int)ceil_div(a.Cout, small ? 32 : 8);
            const long n = (long)a.tiles_xy * a.co_groups * o.n;
            if (small) {
                if (nd.p.stride == 1) set_kernel<KID_C3_T8S1>(t, a, n); else set_kernel<KID_C3_T8S2>(t, a, n);
            } else {
                if (nd.p.stride == 1) set_kernel<KID_C3_T16S1>(t, a, n); else set_kernel<KID_C3_T16S2>(t, a, n);
            }
            break;
        }
        // ---- backward operators and the weight update (graphs that train) ----
        case NG_OP_CONV1X1_DGRAD:
        case NG_OP_CONV3X3_DGRAD: {
            const bool c3 = nd.op == NG_OP_CONV3X3_DGRAD;
            const Shape& dy = i0;                                 // [n][Cout][Ho][Wo]; the result has the shape of the forward input
            GemmArgs a{};
            a.a = wf(0), a.b = buf(nd.preds[0]), a.c = buf(v);
            a.Cin = (int)o.c, a.Cout = (int)dy.c, a.H = (int)o.h, a.W = (int)o.w, a.Ho = (int)dy.h, a.Wo = (int)dy.w;
            a.stride = c3 ? nd.p.stride : 1, a.pad = c3 ? nd.p.pad : 0;
            a.M = a.Cin, a.K = a.Cout * (c3 ? 9 : 1), a.N = (int)(o.n * o.h * o.w);
            a.tiles_n = (int)ceil_div(a.N, kGemmTile), a.splits = 1, a.k_per_split = a.K;
            const long n = (long)a.tiles_n * ceil_div(a.M, kGemmTile);
            if (!c3 && o.h * o.w == 1 && (long)a.M * a.N <= kSmallGemmOutputs && a.K <= kSmallGemmK) {
                // dX[n][ci] = sum_co W[co][ci] dY[n][co]
                SmallGemmArgs sg{a.a, a.b, a.c, nullptr, a.M, a.N, a.K, 1, a.M, 1, a.K, 1, a.M, 0};
                set_small_gemm(t, sg, [](Task& tt, const SmallGemmArgs& aa, long n2) { set_kernel<KID_SMALL_GEMM>(tt, aa, n2); });
                break;
            }
            if (c3) set_kernel<KID_GEMM_C3_DGRAD>(t, a, n);
            else if (pw_px_applies(a)) set_kernel<KID_PW_PX_DGRAD>(t, a, pw_px_tiles(a));
            else set_kernel<KID_GEMM_PW_DGRAD>(t, a, n);
            break;
        }
        case NG_OP_CONV1X1_WGRAD:
        case NG_OP_CONV3X3_WGRAD: {
            const bool c3 = nd.op == NG_OP_CONV3X3_WGRAD;
            const Shape& dy = i0;
            const Shape& x = g->nodes[nd.preds[1]].out;
            GemmArgs a{};
            a.a = buf(nd.preds[0]), a.b = buf(nd.preds[1]), a.c = buf(v);
            a.Cin = (int)x.c, a.Cout = (int)dy.c, a.H = (int)x.h, a.W = (int)x.w, a.Ho = (int)dy.h, a.Wo = (int)dy.w;
            a.stride = c3 ? nd.p.stride : 1, a.pad = c3 ? nd.p.pad : 0;
            a.M = a.Cout, a.N = a.Cin * (c3 ? 9 : 1), a.K = (int)(dy.n * dy.h * dy.w);
            a.tiles_n = (int)ceil_div(a.N, kGemmTile);
            const WgradPlan p = wgrad_plan(g, v);
            a.splits = p.splits, a.k_per_split = p.k_per_split;
            const long tiles = p.tiles;
            if (a.splits > 1) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no workspace for the split-K partial tiles", v);
                a.ws = packed;
                a.cnt = reinterpret_cast<unsigned*>(packed + p.ws_floats);
            }
            if (p.small) {
                // dW[co][ci] = sum_n dY[n][co] X[n][ci]
                SmallGemmArgs sg{a.a, a.b, a.c, nullptr, a.M, a.N, a.K, 1, a.M, a.N, 1, a.N, 1, 0};
                set_small_gemm(t, sg, [](Task& tt, const SmallGemmArgs& aa, long n2) { set_kernel<KID_SMALL_GEMM>(tt, aa, n2); });
                break;
            }
            if (p.px) a.tiles_n = (int)ceil_div(ceil_div(a.N, 16), p.block);
            if (p.px && c3 && p.block == 1) set_kernel<KID_C3_WGRAD_PX>(t, a, tiles * a.splits);
            else if (p.px && c3) set_kernel<KID_C3_WGRAD_PX2>(t, a, tiles * a.splits);
            else if (p.px && p.block == 1) set_kernel<KID_PW_WGRAD_PX>(t, a, tiles * a.splits);
            else if (p.px) set_kernel<KID_PW_WGRAD_PX2>(t, a, tiles * a.splits);
            else if (c3) set_kernel<KID_GEMM_C3_WGRAD>(t, a, tiles * a.splits);
            else set_kernel<KID_GEMM_PW_WGRAD>(t, a, tiles * a.splits);
            break;
        }
        case NG_OP_BN_ACT_DGRAD:
        case NG_OP_BN_ACT_WGRAD: {
            const Shape& x = g->nodes[nd.preds[1]].out;
            BnRawArgs a{};
            a.dy = buf(nd.preds[0]), a.x = buf(nd.preds[1]), a.y = buf(v);
            a.gamma = wf(0), a.beta = wf(1), a.mean = wf(2), a.var = wf(3);
            a.eps = nd.p.eps, a.relu = nd.p.relu != 0;
            a.C = (int)x.c, a.HW = (int)(x.h * x.w), a.N = (int)x.n, a.total = (int)x.elems();
            if (nd.op == NG_OP_BN_ACT_DGRAD) {
                set_kernel<KID_BN_DGRAD>(t, a, ceil_div(a.total, kBlock));
                break;
            }
            a.chunks = (int)bn_wgrad_chunks(a.C, a.N);
            if (a.chunks > 1) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no workspace for the per-chunk sums", v);
                a.ws = packed;
                a.cnt = reinterpret_cast<unsigned*>(packed + (((size_t)a.C * a.chunks * 2 + 63) & ~(size_t)63));
            }
            set_kernel<KID_BN_WGRAD>(t, a, (long)a.C * a.chunks);
            break;
        }
        case NG_OP_RELU_DGRAD:
        case NG_OP_GAP_DGRAD:
        case NG_OP_SLICE_PAD:
        case NG_OP_CHANNEL_SUM: {
            EltGradArgs a{};
            a.dy = buf(nd.preds[0]), a.x = nd.preds.size() > 1 ? buf(nd.preds[1]) : nullptr, a.y = buf(v);
            a.C = (int)o.c, a.HW = hw_out, a.N = (int)o.n, a.total = total;
            if (nd.op == NG_OP_RELU_DGRAD) {
                set_kernel<KID_RELU_DGRAD>(t, a, ceil_div(total, kBlock));
            } else if (nd.op == NG_OP_GAP_DGRAD) {
                a.scale = 1.f / (float)hw_out;
                set_kernel<KID_GAP_DGRAD>(t, a, ceil_div(total, kBlock));
            } else if (nd.op == NG_OP_SLICE_PAD) {
                a.src_C = (int)i0.c, a.src_lo = nd.p.slice_lo[0], a.cnt = nd.p.slice_hi[0] - nd.p.slice_lo[0], a.dst_lo = nd.p.slice_lo[1];
                set_kernel<KID_SLICE_PAD>(t, a, ceil_div(total, kBlock));
            } else {                                              // sums run over the input's images and pixels
                a.C = (int)i0.c, a.HW = (int)(i0.h * i0.w), a.N = (int)i0.n;
                set_kernel<KID_CHANNEL_SUM>(t, a, a.C);
            }
            break;
        }
        case NG_OP_DWCONV_DGRAD:
        case NG_OP_DWCONV_WGRAD: {
            const Shape& dy = i0;
            const Shape& x = g->nodes[nd.preds[1]].out;
            DwGradArgs a{};
            a.dy = buf(nd.preds[0]), a.x = buf(nd.preds[1]), a.y = buf(v);
            a.N = (int)x.n, a.C = (int)x.c, a.H = (int)x.h, a.W = (int)x.w, a.Ho = (int)dy.h, a.Wo = (int)dy.w;
            a.K = nd.p.k, a.S = nd.p.stride, a.total = (int)x.elems();
            if (nd.op == NG_OP_DWCONV_DGRAD) {
                a.w = wf(0);
                const long plane = (long)a.H * a.W, planes = a.total / plane;
                const long quads = a.H * ceil_div(a.W, 4);
                // planes of dx of at most 256 quads; their dy planes, which are no larger, in LDS
                const long per_wg = quads <= kBlock ? std::min<long>(kBlock / quads, (kSmemFloats - kPlaneSlack) / plane_floats(a.Ho, a.Wo, a.K)) : 0;
                const bool whole = a.W % 4 == 0 && a.Wo % 4 == 0;
                if ((a.K == 3 || a.K == 5) && (a.S == 1 || a.S == 2) && a.W >= 4 && a.Wo >= 4 && per_wg > 0 &&
                    a.Ho * ceil_div(a.Wo, 4) <= quads && (whole || a.total >= kRaggedMinElements)) {
                    a.chunks = (int)per_wg;                        // whole planes of dx per workgroup, their dy staged in LDS
                    set_kernel<KID_DW_DGRAD_LDS>(t, a, ceil_div(planes, per_wg));
                    break;
                }
                set_kernel<KID_DW_DGRAD>(t, a, ceil_div(a.total, kBlock));
            } else {
                a.chunks = (int)dw_wgrad_chunks(a.C, a.N);
                if (a.chunks > 1) {
                    if (!packed) return g->fail(NG_EINVAL, "node %d: no workspace for the per-chunk partial sums", v);
                    a.ws = packed;
                    a.cnt = reinterpret_cast<unsigned*>(packed + (((size_t)a.C * a.chunks * a.K * a.K + 63) & ~(size_t)63));
                }
                set_kernel<KID_DW_WGRAD>(t, a, (long)a.C * a.chunks);
            }
            break;
        }
        case NG_OP_POOL_DGRAD: {
            const Shape& dy = i0;
            const Shape& x = g->nodes[nd.preds[1]].out;
            PoolGradArgs a{buf(nd.preds[0]), buf(nd.preds[1]), buf(v), (int)x.h, (int)x.w, (int)dy.h, (int)dy.w,
                           nd.p.stride, nd.p.pad, nd.p.pool_mode, (int)x.elems()};
            const long plane = (long)x.h * x.w;
            if (plane <= kPoolGradChunk && dy.h * dy.w <= plane) {      // whole planes fit a workgroup's LDS
                a.planes_per_tile = (int)(kPoolGradChunk / plane);
                set_kernel<KID_POOL_DGRAD_LDS>(t, a, ceil_div(a.total / plane, a.planes_per_tile));
            } else {
                set_kernel<KID_POOL_DGRAD>(t, a, ceil_div(a.total, kBlock));
            }
            break;
        }
        case NG_OP_SGD_UPDATE: {
            SgdArgs a{};
            a.w = const_cast<float*>(wf(0));                      // caller-owned, updated in place
            a.g = buf(nd.preds[0]), a.flag = buf(v);
            a.lr = nd.p.lr, a.offset = nd.p.slice_lo[0], a.total = nd.p.cout;
            set_kernel<KID_SGD>(t, a, ceil_div(a.total, kBlock));
            break;
        }
        case NG_OP_HEAD_ROPE:
        case NG_OP_HEAD_ROPE_DGRAD:
        case NG_OP_HEAD_ROPE_WGRAD: {
            const RopePlan p = rope_plan(g, v);
            const bool backward = nd.op != NG_OP_HEAD_ROPE, wgrad = nd.op == NG_OP_HEAD_ROPE_WGRAD;
            const int first = backward ? 1 : 0;
            const Shape &x = g->nodes[nd.preds[first]].out, &pos = g->nodes[nd.preds[first + 1]].out;
            RopeArgs a{};
            a.x = buf(nd.preds[first]), a.pos = buf(nd.preds[first + 1]);
            if (backward) a.dy = buf(nd.preds[0]);
            a.freq = wf(0), a.gamma = nd.weights.size() > 1 ? wf(1) : nullptr;
            a.y = buf(v), a.dg = buf(v);
            if (wgrad) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no workspace", v);
                a.ws = packed, a.cnt = reinterpret_cast<unsigned*>(packed + p.ws_floats);
            }
            a.eps = nd.p.eps, a.factor = nd.p.factor;
            a.N = (int)x.n, a.H = nd.p.heads, a.d = (int)(x.c / nd.p.heads), a.T = (int)(x.h * x.w), a.rot = nd.p.rot, a.interleaved = nd.p.interleaved;
            a.pos_stride = pos.n == 1 ? 0 : a.T;
            a.blocks = p.blocks, a.heads_per_tile = p.heads_per_tile, a.items = p.items, a.per_tile = p.per_tile, a.tiles = (int)p.tiles;
            set_any_kernel(t, p.kid, a, p.tiles);
            break;
        }
        case NG_OP_ATTENTION_ROWS: {
            const int y = nd.preds[1];
            const Node& fwd = g->nodes[y];
            const AttentionPlan p = attention_plan(g, y);
            AttnArgs a{};
            a.dy = buf(nd.preds[0]), a.q = buf(y), a.y = buf(v);
            if (!g->packed_of.empty()) a.stats = g->packed_of[y] + p.ws_floats + p.cnt_words;
            a.N = (int)fwd.out.n, a.H = fwd.p.heads, a.d = (int)(fwd.out.c / fwd.p.heads), a.Tq = (int)(fwd.out.h * fwd.out.w);
            set_kernel<KID_ATTN_ROWS>(t, a, (long)a.N * a.H * ceil_div(a.Tq, 64));
            break;
        }
        case NG_OP_ATTENTION:
        case NG_OP_ATTENTION_DQ:
        case NG_OP_ATTENTION_DK:
        case NG_OP_ATTENTION_DV:
        case NG_OP_ATTENTION_DBIAS: {
            const AttentionPlan p = attention_plan(g, v);
            const int first = nd.op == NG_OP_ATTENTION ? 0 : 2;
            const Shape &q = g->nodes[nd.preds[first]].out, &k = g->nodes[nd.preds[first + 1]].out;
            AttnArgs a{};
            a.q = buf(nd.preds[first]), a.k = buf(nd.preds[first + 1]), a.v = buf(nd.preds[first + 2]);
            if ((int)nd.preds.size() == first + 4 + (nd.p.bias != 0)) a.len = buf(nd.preds[first + 3]);
            if (nd.p.bias != 0) {
                const Shape& bias = g->nodes[nd.preds.back()].out;
                a.bias = buf(nd.preds.back()), a.reach = (int)((bias.h * bias.w - 1) / 2), a.from_last = nd.p.bias == 2, a.query_blocks = p.query_blocks;
            }
            if (first) a.dy = buf(nd.preds[0]), a.rows = buf(nd.preds[1]);
            a.y = buf(v);
            if (p.ws_floats + p.stats_floats > 0 && !packed) return g->fail(NG_EINVAL, "node %d: no workspace", v);
            if (nd.op == NG_OP_ATTENTION_DBIAS) a.db = buf(v), a.db_ws = packed, a.db_cnt = reinterpret_cast<unsigned*>(packed + p.ws_floats);
            else if (p.splits > 1) a.ws = packed, a.cnt = reinterpret_cast<unsigned*>(packed + p.ws_floats);
            if (p.stats_floats > 0) a.stats = packed + p.ws_floats + p.cnt_words;
            a.scale = nd.p.scale, a.scale_log2 = (float)((double)nd.p.scale * 1.4426950408889634074);
            a.N = (int)q.n, a.H = nd.p.heads, a.Hk = nd.p.kv_heads, a.d = (int)(q.c / nd.p.heads), a.Tq = (int)(q.h * q.w), a.Tk = (int)(k.h * k.w);
            a.col_blocks = p.col_blocks, a.splits = p.splits, a.per_split = p.per_split;
            set_any_kernel(t, p.kid, a, p.tiles);
            break;
        }
        case NG_OP_LAYER_NORM:
        case NG_OP_LAYER_NORM_DGRAD:
        case NG_OP_LAYER_NORM_WGRAD: {
            const NormPlan p = norm_plan(g, v);
            const bool backward = nd.op != NG_OP_LAYER_NORM;
            const int first = backward ? 1 : 0;
            const Shape& x = g->nodes[nd.preds[first]].out;
            NormArgs a{};
            a.x = buf(nd.preds[first]);
            a.dy = backward ? buf(nd.preds[0]) : a.x;
            a.gamma = wf(0), a.beta = wf(1);
            a.y = buf(v), a.dg = buf(v);
            if (p.cnt_words > 0) {
                if (!packed) return g->fail(NG_EINVAL, "node %d: no workspace", v);
                a.ws = packed, a.cnt = reinterpret_cast<unsigned*>(packed + p.ws_floats);
            }
            a.eps = nd.p.eps, a.C = (int)x.c, a.T = (int)(x.h * x.w);
            a.lanes_log2 = p.lanes_log2, a.blocks = p.blocks, a.items = p.items, a.per_tile = p.per_tile, a.tiles = (int)p.tiles;
            if (norm_channels(p.kid, p.lanes_log2) < x.c) return g->fail(NG_EINVAL, "node %d: the norm's kernel does not hold %lld channels", v, (long long)x.c);
            set_any_kernel(t, p.kid, a, p.tiles);
            break;
        }
        case NG_OP_DROPOUT: {
            DropoutArgs a{};
            a.x = buf(nd.preds[0]), a.seed = buf(nd.preds[1]), a.y = buf(v);
            if (nd.preds.size() > 2) a.residual = buf(nd.preds[2]);
            const double limit = std::nearbyint((double)nd.p.rate * 4294967296.0);
            a.total = o.elems(), a.site = (unsigned)nd.p.site, a.limit = (unsigned)limit, a.scale = (float)(4294967296.0 / (4294967296.0 - limit));
            set_kernel<KID_DROPOUT>(t, a, ceil_div(a.total, kDropoutTile));
            break;
        }
        case NG_OP_POSITION_BIAS:
        case NG_OP_POSITION_BIAS_WGRAD: {
            const bool wgrad = nd.op == NG_OP_POSITION_BIAS_WGRAD;
            if (!packed) return g->fail(NG_EINVAL, "node %d: no buffer for the buckets", v);
            PositionBiasArgs a{};
            if (wgrad) a.dbias = buf(nd.preds[0]);
            else a.table = wf(0);
            a.bucket_of = reinterpret_cast<const int*>(packed), a.out = buf(v);
            a.heads = nd.p.heads, a.distances = 2 * nd.p.max_distance + 1, a.buckets = nd.p.buckets;
            if (wgrad) set_kernel<KID_POSITION_BIAS_WGRAD>(t, a, ceil_div((long)a.buckets * a.heads, kBlock / 64));
            else set_kernel<KID_POSITION_BIAS>(t, a, ceil_div((long)a.heads * a.distances, kBlock));
            break;
        }
        default:
            return g->fail(NG_EINVAL, "node %d: operator %d has no kernel", v, nd.op);
    }
    if (t.ntiles <= 0 || t.ntiles >= (1L << 31)) return g->fail(NG_ESHAPE, "node %d: %ld tiles cannot be launched", v, t.ntiles);
    return NG_OK;
}

}  // namespace ng
