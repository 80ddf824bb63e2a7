// C ABI of the low-rank adapters (include/pp_adapter.h): the bank, checks, launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "adapter_rules.hpp"
#include "block_plan.hpp"
#include "k8_adapter.hpp"
#include "pp_adapter.h"

struct pp_adapter_bank {
    int m = 0, k = 0, slots = 0, max_rank = 0, rank_pad = 0, dtype = PP_F32;
    bool on_device = false;
    int device = 0;
    // one allocation: ranks, factors, then the operands of all slots in four orders
    void* memory = nullptr;
    int32_t* rank = nullptr;
    float* scale = nullptr;
    char *a_project = nullptr, *b_project = nullptr, *a_expand = nullptr, *b_expand = nullptr;
    // bytes of one slot in each
    int64_t a_project_slot = 0, b_project_slot = 0, a_expand_slot = 0, b_expand_slot = 0;
};

namespace {

using namespace ppc;

struct Range {
    uintptr_t from = 0, to = 0;
    Range(const void* p, int64_t bytes) : from(reinterpret_cast<uintptr_t>(p)), to(from + (uintptr_t)bytes) {}
};
bool overlap(const Range& a, const Range& b) { return a.from < b.to && b.from < a.to; }
bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
int64_t elem(const pp_adapter_bank_t* b) { return b->dtype == PP_F16 ? 2 : 4; }

bool tokens_ok(const pp_adapter_bank_t* b, int32_t n) {
    return n >= 1 && n <= kAdapterMaxTokens && (int64_t)b->k * n < ((int64_t)1 << 31) && (int64_t)b->m * n < ((int64_t)1 << 31);
}
pp_status_t ready(const pp_adapter_bank_t* b) {
    if (!b->on_device) return PP_ERR_UNSUPPORTED;
    int device = -1;
    return hipGetDevice(&device) == hipSuccess && device == b->device ? PP_OK : PP_ERR_DEVICE;
}
pp_status_t plan_fits(const pp_adapter_bank_t* b, const pp_block_gemm_plan_t* plan, bool transposed, int32_t n) {
    const BlockPlanFacts f = block_plan_facts(plan);
    if (f.dtype != b->dtype) return PP_ERR_UNSUPPORTED;
    if (f.m != (transposed ? b->k : b->m) || f.k != (transposed ? b->m : b->k) || f.transposed != transposed) return PP_ERR_SHAPE;
    const pp_status_t st = block_check_adapted(plan, n);
    if (st != PP_OK) return st;
    return !b->on_device || f.device == b->device ? PP_OK : PP_ERR_DEVICE;
}

// ---- launches (everything has been checked) ----

// n <= N slots, none twice, ranks up to `top`
template <typename T, int N>
void load_slots(const pp_adapter_bank_t* b, int n, int top, const int32_t* slot, const int32_t* rank, const float* scale, const void* const* a_dev,
                const void* const* b_dev, hipStream_t stream) {
    K8Load<N> p{};
    p.a_project = b->a_project, p.b_project = b->b_project, p.a_expand = b->a_expand, p.b_expand = b->b_expand;
    const int64_t eb = elem(b);
    p.a_project_slot = b->a_project_slot / eb, p.b_project_slot = b->b_project_slot / eb;
    p.a_expand_slot = b->a_expand_slot / eb, p.b_expand_slot = b->b_expand_slot / eb;
    p.rank = b->rank, p.scale = b->scale;
    p.m = b->m, p.k = b->k, p.rank_pad = b->rank_pad;
    for (int i = 0; i < n; ++i) p.of[i] = K8LoadSlot{a_dev[i], b_dev[i], scale[i], rank[i], slot[i], 0};
    const int pad = adapter_rank_pad(top);
    const bool half = sizeof(T) == 2;
    const int64_t items = (adapter_project_elems(b->k, pad) + adapter_project_elems(b->m, pad) + adapter_expand_elems(b->k, pad, half) +
                           adapter_expand_elems(b->m, pad, half)) / 8, wgs = (items + 255) / 256;
    const unsigned grid = wgs < 1 ? 1u : (wgs < 65536 ? (unsigned)wgs : 65536u);
    hipLaunchKernelGGL((k8_load_slots<T, N>), dim3(grid, (unsigned)n), dim3(256), 0, stream, p);
}

template <typename T, int FT, int RG, bool GATED> void project_as(const K8Project& a, dim3 grid, hipStream_t stream) {
    hipLaunchKernelGGL((k8_project<T, FT, RG, GATED>), grid, dim3(64 * kProjectWaves), 0, stream, a);
}
template <typename T, int FT, bool GATED> void project_rg(const K8Project& a, dim3 grid, hipStream_t stream) {
    constexpr int most = sizeof(T) == 4 && FT == 4 ? 2 : 4;      // rank tiles in registers at a time: four would spill there
    if (a.rank_pad <= 16) project_as<T, FT, 1, GATED>(a, grid, stream);
    else if (a.rank_pad <= 32) project_as<T, FT, 2, GATED>(a, grid, stream);
    else project_as<T, FT, most, GATED>(a, grid, stream);
}
template <typename T, bool GATED> void project_ft(int ft, const K8Project& a, dim3 grid, hipStream_t stream) {
    if (ft == 1) project_rg<T, 1, GATED>(a, grid, stream);
    else if (ft == 2) project_rg<T, 2, GATED>(a, grid, stream);
    else project_rg<T, 4, GATED>(a, grid, stream);
}

// where the sums of what a projection left start
float* sums_of(void* state, int n) { return reinterpret_cast<float*>(static_cast<KxToken*>(state) + n); }
const float* sums_of(const void* state, int n) { return reinterpret_cast<const float*>(static_cast<const KxToken*>(state) + n); }

// u = A x (of_a) or v = B^T x
void launch_project(const pp_adapter_bank_t* b, bool of_a, const void* x, const void* gate, void* g, const int32_t* slot_of, void* u, int n, hipStream_t stream) {
    K8Project a{};
    a.rows = of_a ? b->k : b->m;
    const ProjectShape sh = project_shape(a.rows, n, b->dtype == PP_F16, !of_a);
    a.x = x, a.gate = static_cast<const int8_t*>(gate), a.g = g, a.slot_of = slot_of, a.rank = b->rank, a.scale = b->scale;
    a.tokens = static_cast<KxToken*>(u), a.u = sums_of(u, n);
    a.operands = of_a ? b->a_project : b->b_project;
    a.slot_elems = (of_a ? b->a_project_slot : b->b_project_slot) / elem(b);
    a.gate_pitch = act8_pitch(n);
    a.n = n, a.steps = (a.rows + 31) / 32, a.slots = b->slots, a.rank_pad = b->rank_pad, a.splits = sh.splits;
    const dim3 grid((unsigned)(sh.tiles * sh.splits), (unsigned)project_subsets(sh, b->slots));
    if (b->dtype == PP_F16) {
        if (gate) project_ft<_Float16, true>(sh.ft, a, grid, stream);
        else project_ft<_Float16, false>(sh.ft, a, grid, stream);
    } else {
        if (gate) project_ft<float, true>(sh.ft, a, grid, stream);
        else project_ft<float, false>(sh.ft, a, grid, stream);
    }
}

// y = act(W x + bias + c B u) with the plan's W, bias and act (of_b), or with A^T in place of B
pp_status_t launch_product(const pp_adapter_bank_t* b, bool of_b, const pp_block_gemm_plan_t* plan, const void* x, const void* u, void* y, int n,
                           hipStream_t stream) {
    const int rows_in = of_b ? b->k : b->m;
    const int splits = project_shape(rows_in, n, b->dtype == PP_F16, !of_b).splits;
    const int64_t split_elems = kx_share(n, b->rank_pad);
    if (b->dtype == PP_F16) {
        K4Expand e{};
        e.tokens = static_cast<const KxToken*>(u), e.u = sums_of(u, n);
        e.operands = of_b ? b->b_expand : b->a_expand;
        e.slot_bytes = of_b ? b->b_expand_slot : b->a_expand_slot;
        e.split_elems = split_elems;
        e.splits = splits, e.rank_pad = b->rank_pad;
        return block_launch_adapted(plan, x, y, n, e, stream);
    }
    const pp_status_t st = block_launch_linear_f32(plan, x, y, n, stream);
    if (st != PP_OK) return st;
    K8Expand a{};
    a.y = static_cast<float*>(y), a.tokens = static_cast<const KxToken*>(u), a.u = sums_of(u, n);
    a.operands = reinterpret_cast<const float*>(of_b ? b->b_expand : b->a_expand);
    a.slot_elems = (of_b ? b->b_expand_slot : b->a_expand_slot) / 4;
    a.split_elems = split_elems;
    a.m = of_b ? b->m : b->k, a.n = n, a.splits = splits, a.rank_pad = b->rank_pad, a.relu = block_plan_facts(plan).relu;
    const bool few = expand_few(a.m, n, b->slots);
    const int token_tiles = few ? (n + 15) / 16 : (n + 63) / 64;
    const dim3 grid((unsigned)(few ? (a.m + 15) / 16 : (a.m + 63) / 64), (unsigned)(token_tiles < 32768 ? token_tiles : 32768));
    if (few) hipLaunchKernelGGL(k8_expand_few, grid, dim3(64 * kExpandWaves), 0, stream, a);
    else hipLaunchKernelGGL(k8_expand_f32, grid, dim3(256), 0, stream, a);
    return PP_OK;
}

template <typename T, bool HELD8> void launch_grad(int rw, const K8Grad& a, dim3 grid, hipStream_t stream) {
    if (a.rank_pad <= 16) hipLaunchKernelGGL((k8_grad<T, 1, 1, HELD8>), grid, dim3(256), 0, stream, a);
    else if (a.rank_pad <= 32) hipLaunchKernelGGL((k8_grad<T, 2, 1, HELD8>), grid, dim3(256), 0, stream, a);
    else if (rw == 1) hipLaunchKernelGGL((k8_grad<T, 4, 1, HELD8>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((k8_grad<T, 4, 2, HELD8>), grid, dim3(256), 0, stream, a);
}

pp_status_t launched() { return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_DEVICE; }

}  // namespace

extern "C" {

pp_status_t pp_adapter_plan(const pp_adapter_desc_t* desc, pp_adapter_bank_t** out_bank) {
    if (out_bank) *out_bank = nullptr;
    if (!desc || !out_bank) return PP_ERR_NULL;
    if (desc->m < 1 || desc->k < 1 || (int64_t)desc->m * desc->k >= ((int64_t)1 << 31)) return PP_ERR_SHAPE;
    if (desc->m > kAdapterMaxRows || desc->k > kAdapterMaxRows) return PP_ERR_SHAPE;
    if (desc->slots < 1 || desc->slots > kAdapterMaxSlots || desc->max_rank < 1 || desc->max_rank > kAdapterMaxRank) return PP_ERR_SHAPE;
    if (desc->dtype != PP_F32 && desc->dtype != PP_F16) return PP_ERR_UNSUPPORTED;
    if (desc->flags & ~(uint32_t)PP_FLAG_HOST_ONLY) return PP_ERR_UNSUPPORTED;
    pp_adapter_bank_t* b = new (std::nothrow) pp_adapter_bank_t();
    if (!b) return PP_ERR_ALLOC;
    b->m = desc->m, b->k = desc->k, b->slots = desc->slots, b->max_rank = desc->max_rank, b->dtype = desc->dtype;
    b->rank_pad = adapter_rank_pad(desc->max_rank);
    const int64_t eb = elem(b);
    const bool half = desc->dtype == PP_F16;
    b->a_project_slot = adapter_project_elems(b->k, b->rank_pad) * eb;
    b->b_project_slot = adapter_project_elems(b->m, b->rank_pad) * eb;
    b->a_expand_slot = adapter_expand_elems(b->k, b->rank_pad, half) * eb;
    b->b_expand_slot = adapter_expand_elems(b->m, b->rank_pad, half) * eb;
    if (!(desc->flags & PP_FLAG_HOST_ONLY)) {
        const int64_t table = ((int64_t)b->slots * 4 + 255) / 256 * 256;
        const int64_t slot = b->a_project_slot + b->b_project_slot + b->a_expand_slot + b->b_expand_slot;
        void* p = nullptr;
        if (hipGetDevice(&b->device) != hipSuccess || hipMalloc(&p, (size_t)(2 * table + slot * b->slots)) != hipSuccess ||
            hipMemset(p, 0, (size_t)(2 * table)) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
            (void)hipGetLastError();
            if (p) (void)hipFree(p);
            delete b;
            return PP_ERR_DEVICE;
        }
        b->memory = p;
        char* at = static_cast<char*>(p);
        b->rank = reinterpret_cast<int32_t*>(at), at += table;
        b->scale = reinterpret_cast<float*>(at), at += table;
        b->a_project = at, at += b->a_project_slot * b->slots;
        b->b_project = at, at += b->b_project_slot * b->slots;
        b->a_expand = at, at += b->a_expand_slot * b->slots;
        b->b_expand = at;
        b->on_device = true;
    }
    *out_bank = b;
    return PP_OK;
}

pp_status_t pp_adapter_load_many(pp_adapter_bank_t* bank, int32_t count, const int32_t* slot, const int32_t* rank, const float* scale,
                                 const void* const* a_dev, const void* const* b_dev, void* hip_stream) {
    if (!bank || !slot || !rank || !scale || !a_dev || !b_dev) return PP_ERR_NULL;
    if (count < 1) return PP_ERR_SHAPE;
    for (int32_t i = 0; i < count; ++i) {
        if (rank[i] != 0 && (!a_dev[i] || !b_dev[i])) return PP_ERR_NULL;
        if (slot[i] < 0 || slot[i] >= bank->slots || rank[i] < 0 || rank[i] > bank->max_rank) return PP_ERR_SHAPE;
        if (!std::isfinite(scale[i])) return PP_ERR_UNSUPPORTED;
        if (rank[i] && (misaligned(a_dev[i]) || misaligned(b_dev[i]))) return PP_ERR_ALIGN;
    }
    const pp_status_t st = ready(bank);
    if (st != PP_OK) return st;
    (void)hipGetLastError();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    for (int32_t from = 0; from < count;) {
        // up to kAdapterLoads slots, none of them twice: their loads have no order within a launch
        int n = 0, top = 0;
        for (; n < kAdapterLoads && from + n < count; ++n) {
            bool again = false;
            for (int i = 0; i < n; ++i) again = again || slot[from + i] == slot[from + n];
            if (again) break;
            top = rank[from + n] > top ? rank[from + n] : top;
        }
        if (bank->dtype == PP_F16) {
            if (n == 1) load_slots<_Float16, 1>(bank, 1, top, slot + from, rank + from, scale + from, a_dev + from, b_dev + from, stream);
            else load_slots<_Float16, kAdapterLoads>(bank, n, top, slot + from, rank + from, scale + from, a_dev + from, b_dev + from, stream);
        } else {
            if (n == 1) load_slots<float, 1>(bank, 1, top, slot + from, rank + from, scale + from, a_dev + from, b_dev + from, stream);
            else load_slots<float, kAdapterLoads>(bank, n, top, slot + from, rank + from, scale + from, a_dev + from, b_dev + from, stream);
        }
        from += n;
    }
    return launched();
}

pp_status_t pp_adapter_load(pp_adapter_bank_t* bank, int32_t slot, int32_t rank, float scale, const void* a_dev, const void* b_dev, void* hip_stream) {
    return pp_adapter_load_many(bank, 1, &slot, &rank, &scale, &a_dev, &b_dev, hip_stream);
}

int64_t pp_adapter_u_bytes(const pp_adapter_bank_t* bank, int32_t n) { return bank && tokens_ok(bank, n) ? adapter_state_bytes(bank->k, n, bank->rank_pad, bank->dtype == PP_F16, false) : 0; }
int64_t pp_adapter_v_bytes(const pp_adapter_bank_t* bank, int32_t n) { return bank && tokens_ok(bank, n) ? adapter_state_bytes(bank->m, n, bank->rank_pad, bank->dtype == PP_F16, true) : 0; }
int64_t pp_adapter_work_bytes(const pp_adapter_bank_t* bank, int32_t n, int32_t count) {
    return bank && tokens_ok(bank, n) && count >= 1 && count <= 65535 ? grad_work(bank->m, bank->k, n, count, bank->rank_pad, bank->dtype == PP_F16).bytes : 0;
}

pp_status_t pp_adapter_project(const pp_adapter_bank_t* bank, const void* x_dev, const int32_t* slot_of_dev, void* u_dev, int32_t n, void* hip_stream) {
    if (!bank || !x_dev || !slot_of_dev || !u_dev) return PP_ERR_NULL;
    if (!tokens_ok(bank, n)) return PP_ERR_SHAPE;
    if (misaligned(x_dev) || misaligned(u_dev) || misaligned4(slot_of_dev)) return PP_ERR_ALIGN;
    const Range x(x_dev, (int64_t)bank->k * n * elem(bank)), u(u_dev, pp_adapter_u_bytes(bank, n)), s(slot_of_dev, (int64_t)n * 4);
    if (overlap(u, x) || overlap(u, s)) return PP_ERR_ALIGN;
    const pp_status_t st = ready(bank);
    if (st != PP_OK) return st;
    (void)hipGetLastError();
    launch_project(bank, true, x_dev, nullptr, nullptr, slot_of_dev, u_dev, n, static_cast<hipStream_t>(hip_stream));
    return launched();
}

pp_status_t pp_adapter_run(const pp_adapter_bank_t* bank, const pp_block_gemm_plan_t* plan, const void* x_dev, const int32_t* slot_of_dev, void* u_dev,
                           void* y_dev, int32_t n, void* hip_stream) {
    if (!bank || !plan || !x_dev || !slot_of_dev || !u_dev || !y_dev) return PP_ERR_NULL;
    if (!tokens_ok(bank, n)) return PP_ERR_SHAPE;
    if (misaligned(x_dev) || misaligned(u_dev) || misaligned(y_dev) || misaligned4(slot_of_dev)) return PP_ERR_ALIGN;
    const Range x(x_dev, (int64_t)bank->k * n * elem(bank)), y(y_dev, (int64_t)bank->m * n * elem(bank)), u(u_dev, pp_adapter_u_bytes(bank, n)),
        s(slot_of_dev, (int64_t)n * 4);
    if (overlap(u, x) || overlap(u, s) || overlap(y, x) || overlap(y, u) || overlap(y, s)) return PP_ERR_ALIGN;
    pp_status_t st = plan_fits(bank, plan, false, n);
    if (st == PP_OK) st = ready(bank);
    if (st != PP_OK) return st;
    (void)hipGetLastError();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    launch_project(bank, true, x_dev, nullptr, nullptr, slot_of_dev, u_dev, n, stream);
    st = launched();
    if (st != PP_OK) return st;
    st = launch_product(bank, true, plan, x_dev, u_dev, y_dev, n, stream);
    return st == PP_OK ? launched() : st;
}

pp_status_t pp_adapter_grad_input(const pp_adapter_bank_t* bank, const pp_block_gemm_plan_t* plan_t, const void* dy_dev, const void* gate_dev, void* g_dev,
                                  const int32_t* slot_of_dev, void* v_dev, void* dx_dev, int32_t n, void* hip_stream) {
    if (!bank || !dy_dev || !slot_of_dev || !v_dev || (gate_dev && !g_dev) || (dx_dev && !plan_t)) return PP_ERR_NULL;
    if (!tokens_ok(bank, n)) return PP_ERR_SHAPE;
    if (misaligned(dy_dev) || misaligned(v_dev) || misaligned4(slot_of_dev) || (gate_dev && (misaligned(gate_dev) || misaligned(g_dev))) || (dx_dev && misaligned(dx_dev))) return PP_ERR_ALIGN;
    const int64_t out_bytes = (int64_t)bank->m * n * elem(bank);
    const Range dy(dy_dev, out_bytes), v(v_dev, pp_adapter_v_bytes(bank, n)), s(slot_of_dev, (int64_t)n * 4);
    if (overlap(v, dy) || overlap(v, s)) return PP_ERR_ALIGN;
    if (gate_dev) {
        const Range gate(gate_dev, act8_bytes(bank->m, n)), g(g_dev, out_bytes);
        if ((g_dev != dy_dev && overlap(g, dy)) || overlap(g, v) || overlap(g, s) || overlap(g, gate) || overlap(v, gate)) return PP_ERR_ALIGN;
        if (dx_dev) {
            const Range dx(dx_dev, (int64_t)bank->k * n * elem(bank));
            if (overlap(dx, g) || overlap(dx, gate)) return PP_ERR_ALIGN;
        }
    }
    if (dx_dev) {
        const Range dx(dx_dev, (int64_t)bank->k * n * elem(bank));
        if (overlap(dx, dy) || overlap(dx, v) || overlap(dx, s)) return PP_ERR_ALIGN;
    }
    pp_status_t st = dx_dev ? plan_fits(bank, plan_t, true, n) : PP_OK;
    if (st == PP_OK) st = ready(bank);
    if (st != PP_OK) return st;
    (void)hipGetLastError();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    launch_project(bank, false, dy_dev, gate_dev, g_dev, slot_of_dev, v_dev, n, stream);
    st = launched();
    if (st != PP_OK || !dx_dev) return st;
    st = launch_product(bank, false, plan_t, gate_dev ? g_dev : dy_dev, v_dev, dx_dev, n, stream);
    return st == PP_OK ? launched() : st;
}

pp_status_t pp_adapter_grad_weights(const pp_adapter_bank_t* bank, const void* x_dev, int32_t x_is_act8, const void* u_dev, const void* g_dev,
                                    const void* v_dev, const int32_t* slot_of_dev, const int32_t* which_dev, int32_t count, float* da_dev, float* db_dev,
                                    void* work_dev, int32_t n, void* hip_stream) {
    if (!bank || !x_dev || !u_dev || !g_dev || !v_dev || !slot_of_dev || !which_dev || !da_dev || !db_dev || !work_dev) return PP_ERR_NULL;
    if (!tokens_ok(bank, n) || count < 1 || count > 65535) return PP_ERR_SHAPE;
    const void* all[] = {x_dev, u_dev, g_dev, v_dev, da_dev, db_dev, work_dev};
    for (const void* p : all)
        if (misaligned(p)) return PP_ERR_ALIGN;
    if (misaligned4(slot_of_dev) || misaligned4(which_dev)) return PP_ERR_ALIGN;
    const Range in[] = {Range(x_dev, x_is_act8 ? act8_bytes(bank->k, n) : (int64_t)bank->k * n * elem(bank)), Range(u_dev, pp_adapter_u_bytes(bank, n)),
                        Range(g_dev, (int64_t)bank->m * n * elem(bank)), Range(v_dev, pp_adapter_v_bytes(bank, n)), Range(slot_of_dev, (int64_t)n * 4),
                        Range(which_dev, (int64_t)count * 4)};
    const Range out[] = {Range(da_dev, (int64_t)count * bank->max_rank * bank->k * 4), Range(db_dev, (int64_t)count * bank->max_rank * bank->m * 4),
                         Range(work_dev, pp_adapter_work_bytes(bank, n, count))};
    for (int i = 0; i < 3; ++i) {
        for (const Range& r : in)
            if (overlap(out[i], r)) return PP_ERR_ALIGN;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return PP_ERR_ALIGN;
    }
    const pp_status_t st = ready(bank);
    if (st != PP_OK) return st;
    const bool half = bank->dtype == PP_F16;
    const GradShape sh = grad_shape(bank->m, bank->k, n, count, bank->rank_pad, half, x_is_act8 != 0);
    const GradWork at = grad_work(bank->m, bank->k, n, count, bank->rank_pad, half);
    char* work = static_cast<char*>(work_dev);
    K8Turned turned;
    turned.slots = reinterpret_cast<K8Slot*>(work), turned.masks = reinterpret_cast<K8Mask*>(work + at.masks);
    turned.w = work + at.w, turned.down = reinterpret_cast<float*>(work + at.down);
    (void)hipGetLastError();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    K8Turn t{};
    t.out = turned;
    t.w[0] = sums_of(v_dev, n), t.w[1] = sums_of(u_dev, n);
    t.splits[0] = project_shape(bank->m, n, half, true).splits, t.splits[1] = project_shape(bank->k, n, half, false).splits;
    t.tokens[0] = static_cast<const KxToken*>(v_dev), t.tokens[1] = static_cast<const KxToken*>(u_dev);
    t.slot_of = slot_of_dev;
    t.n = n, t.blocks = (n + kAct8Block - 1) / kAct8Block, t.rank_pad = bank->rank_pad, t.x_is_act8 = x_is_act8 ? 1 : 0;
    K8Grad a{};
    a.in = turned;
    a.x = x_dev, a.g = g_dev;
    a.x_pitch = act8_pitch(n), a.x_scale_pitch = act8_scale_pitch(bank->k);
    a.x_scale = x_is_act8 ? static_cast<const uint8_t*>(x_dev) + bank->k * a.x_pitch : nullptr;
    a.work = reinterpret_cast<float*>(work + at.sums);
    a.m = bank->m, a.k = bank->k, a.n = n, a.blocks = t.blocks, a.rank_pad = bank->rank_pad, a.max_rank = bank->max_rank;
    a.tiles_k = sh.tiles_k, a.count = at.batch, a.splits = sh.splits;
    K8Join j{};
    j.slots = turned.slots, j.work = a.work;
    j.m = bank->m, j.k = bank->k, j.rank_pad = bank->rank_pad, j.max_rank = bank->max_rank, j.count = at.batch, j.splits = sh.splits;
    j.wgs_a = ((int64_t)bank->k * bank->max_rank + 255) / 256;
    for (int from = 0; from < count; from += at.batch) {
        const unsigned slots = (unsigned)(count - from < at.batch ? count - from : at.batch);
        t.which = which_dev + from;
        a.da = j.da = da_dev + (int64_t)from * bank->max_rank * bank->k;
        a.db = j.db = db_dev + (int64_t)from * bank->max_rank * bank->m;
        const dim3 turns((unsigned)t.blocks, slots, (unsigned)(2 * (bank->rank_pad / 16)));
        if (half) hipLaunchKernelGGL(k8_turn<_Float16>, turns, dim3(256), 0, stream, t);
        else hipLaunchKernelGGL(k8_turn<float>, turns, dim3(256), 0, stream, t);
        const dim3 grid((unsigned)(sh.tiles_k + sh.tiles_m), slots, (unsigned)sh.splits);
        if (half) {
            if (x_is_act8) launch_grad<_Float16, true>(sh.rw, a, grid, stream);
            else launch_grad<_Float16, false>(sh.rw, a, grid, stream);
        } else {
            if (x_is_act8) launch_grad<float, true>(sh.rw, a, grid, stream);
            else launch_grad<float, false>(sh.rw, a, grid, stream);
        }
        if (sh.splits > 1) {
            const int64_t wgs = j.wgs_a + ((int64_t)bank->m * bank->max_rank + 255) / 256;
            hipLaunchKernelGGL(k8_grad_join, dim3((unsigned)wgs, slots), dim3(256), 0, stream, j);
        }
    }
    return launched();
}

pp_status_t pp_adapter_destroy(pp_adapter_bank_t* bank) {
    if (!bank) return PP_OK;
    if (bank->memory) (void)hipFree(bank->memory);
    delete bank;
    return PP_OK;
}

}  // extern "C"
