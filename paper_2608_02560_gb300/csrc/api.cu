// C ABI of the PRECOG hot path: argument validation, dispatch to the
// kernels, status codes. Nothing here allocates device memory.
#include <atomic>
#include <cstdarg>
#include <map>
#include <mutex>
#include <utility>
#include <cstdio>
#include <cstring>

#include "../../include/precog.h"
#include "internal.h"

namespace {

thread_local char g_last_error[512] = "";

precog_status fail(precog_status s, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return s;
}

precog_status ok() {
    g_last_error[0] = '\0';
    return PRECOG_OK;
}

precog_status cuda_fail(cudaError_t e, const char *what) {
    return fail(PRECOG_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int dtype_size(int32_t dt) {
    switch (dt) {
        case PRECOG_F32: return 4;
        case PRECOG_BF16: return 2;
        case PRECOG_F16: return 2;
        default: return 0;
    }
}

bool state_dtype_ok(int32_t dt) { return dt == PRECOG_F32 || dt == PRECOG_BF16; }

// Checks shared by encode and prefill. rows = T_tot per layer.
precog_status check_scan_inputs(const precog_scan_inputs *in, int64_t rows, bool need_C) {
    if (in == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "scan inputs pointer is NULL");
    if (in->n_layers < 1) return fail(PRECOG_ERR_INVALID_ARG, "n_layers must be >= 1");
    if (in->N != 16) return fail(PRECOG_ERR_UNSUPPORTED, "N=%d: only N=16 is implemented", in->N);
    if (in->D < 1) return fail(PRECOG_ERR_INVALID_ARG, "D must be >= 1");
    if (in->a_kind != PRECOG_A_GENERAL && in->a_kind != PRECOG_A_POWER &&
        in->a_kind != PRECOG_A_COMPLEX)
        return fail(PRECOG_ERR_INVALID_ARG, "a_kind must be PRECOG_A_GENERAL, _POWER or _COMPLEX");
    if (in->in_dtype != PRECOG_F32 && in->in_dtype != PRECOG_BF16)
        return fail(PRECOG_ERR_UNSUPPORTED, "in_dtype must be PRECOG_F32 or PRECOG_BF16");
    const int sz = dtype_size(in->in_dtype);
    if ((static_cast<int64_t>(in->D) * sz) % 16 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "D*sizeof(in_dtype) must be a multiple of 16");
    if (in->A == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "A must be non-NULL");
    if (rows > 0 && (in->x == nullptr || in->dt == nullptr || in->B == nullptr))
        return fail(PRECOG_ERR_INVALID_ARG, "x, dt and B must be non-NULL");
    if (rows > 0 && need_C && in->C == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "C is required when y_out is given");
    if (!aligned16(in->x) || !aligned16(in->dt) || !aligned16(in->B) || !aligned16(in->A) ||
        (in->C && !aligned16(in->C)))
        return fail(PRECOG_ERR_INVALID_ARG, "input pointers must be 16-byte aligned");
    if (in->n_layers > 1) {
        if (in->layer_stride_xd < rows * in->D || in->layer_stride_bc < rows * in->N)
            return fail(PRECOG_ERR_INVALID_ARG, "layer strides smaller than one layer block");
        if ((in->layer_stride_xd * sz) % 16 != 0 || (in->layer_stride_bc * sz) % 16 != 0)
            return fail(PRECOG_ERR_INVALID_ARG, "layer strides must keep 16-byte alignment");
    }
    return PRECOG_OK;
}

precog::ScanParams base_params(const precog_scan_inputs *in, int64_t rows) {
    precog::ScanParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = in->x;
    p.dt = in->dt;
    p.B = in->B;
    p.C = in->C;
    p.A = in->A;
    p.ls_xd = in->n_layers > 1 ? in->layer_stride_xd : 0;
    p.ls_bc = in->n_layers > 1 ? in->layer_stride_bc : 0;
    p.n_layers = in->n_layers;
    p.D = in->D;
    p.N = in->N;
    p.in_dtype = in->in_dtype;
    p.a_kind = in->a_kind;
    p.T_tot = rows;
    return p;
}

// CTAs of one launch.
constexpr int64_t kMaxItems = 0x7fffffffLL;

// Checks shared by the delta rule's scan and step.
precog_status check_delta_inputs(const precog_delta_inputs *in, int64_t rows, bool need_q) {
    if (in == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "delta inputs pointer is NULL");
    if (in->in_dtype != PRECOG_F32 && in->in_dtype != PRECOG_BF16)
        return fail(PRECOG_ERR_UNSUPPORTED, "in_dtype must be PRECOG_F32 or PRECOG_BF16");
    if (in->n_qk_heads < 1 || in->n_v_heads < 1 || in->n_v_heads % in->n_qk_heads != 0)
        return fail(PRECOG_ERR_INVALID_ARG, "n_v_heads must be a positive multiple of n_qk_heads");
    if (in->n_v_heads > 65535) return fail(PRECOG_ERR_UNSUPPORTED, "n_v_heads must be below 2^16");
    if (in->dk < 8 || in->dk > 128 || in->dk % 8 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "dk=%d: a multiple of 8 in [8, 128] is implemented", in->dk);
    if (in->dv < 8 || in->dv > 4096 || in->dv % 8 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "dv=%d: a multiple of 8 in [8, 4096] is implemented", in->dv);
    if (rows == 0) return PRECOG_OK;
    if (in->k == nullptr || in->v == nullptr || in->g == nullptr || in->beta == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "k, v, g and beta must be non-NULL");
    if (need_q && in->q == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "q is required when y_out is given");
    if ((in->q && !aligned16(in->q)) || !aligned16(in->k) || !aligned16(in->v) || !aligned16(in->g) ||
        !aligned16(in->beta))
        return fail(PRECOG_ERR_INVALID_ARG, "input pointers must be 16-byte aligned");
    if (rows > 1) {
        const int sz = dtype_size(in->in_dtype);
        const int64_t row_k = static_cast<int64_t>(in->n_qk_heads) * in->dk;
        const int64_t row_v = static_cast<int64_t>(in->n_v_heads) * in->dv;
        if ((in->q && in->q_stride < row_k) || in->k_stride < row_k || in->v_stride < row_v)
            return fail(PRECOG_ERR_INVALID_ARG, "row strides smaller than a row");
        if ((in->q && (in->q_stride * sz) % 16 != 0) || (in->k_stride * sz) % 16 != 0 || (in->v_stride * sz) % 16 != 0)
            return fail(PRECOG_ERR_INVALID_ARG, "row strides must keep 16-byte alignment");
    }
    return PRECOG_OK;
}

precog::DeltaParams delta_params(const precog_delta_inputs *in) {
    precog::DeltaParams p;
    std::memset(&p, 0, sizeof(p));
    p.q = in->q;
    p.k = in->k;
    p.v = in->v;
    p.g = in->g;
    p.beta = in->beta;
    p.q_stride = in->q_stride;
    p.k_stride = in->k_stride;
    p.v_stride = in->v_stride;
    p.hk = in->n_qk_heads;
    p.hv = in->n_v_heads;
    p.dk = in->dk;
    p.dv = in->dv;
    p.in_dtype = in->in_dtype;
    p.scale = in->scale;
    return p;
}

// The kernel files' status words, taken and cleared at once: a copy of each would wait for the device
// every time (eleven words: 144 us a call, so 22).
constexpr cudaError_t (*kStatusWord[])(uint32_t **) = {
    precog::scan_status_word,    precog::scan_complex_status_word, precog::scan_latency_status_word, precog::retrieve_status_word,
    precog::retrieve_tc_status_word, precog::smc_status_word,      precog::selftest_status_word,     precog::delta_status_word,
    precog::delta_chunk_status_word, precog::qk_norm_status_word,  precog::logprobs_status_word};
constexpr int kStatusWords = sizeof(kStatusWord) / sizeof(kStatusWord[0]);
static_assert(kStatusWords <= 32, "a lane each");
struct StatusWords {
    uint32_t *word[kStatusWords];
};
__device__ uint32_t g_taken_status;
std::mutex g_status_mutex;   // of g_taken_status
__global__ void take_status_kernel(const StatusWords words) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < kStatusWords; ++i)
        if (threadIdx.x == i) bits = atomicExch(words.word[i], 0u);
    bits = __reduce_or_sync(0xffffffffu, bits);
    if (threadIdx.x == 0) g_taken_status = bits;
}

std::atomic<uint64_t> g_launches{0};
std::mutex g_attr_mutex;
// dynamic shared-memory limit already set, per (kernel, device): the attribute is per device
std::map<std::pair<const void *, int>, int> g_smem_attr;

}  // namespace

namespace precog {

void count_launches(uint64_t n) { g_launches.fetch_add(n, std::memory_order_relaxed); }

int device_sm_count() {
    constexpr int kMaxDevices = 64;
    static std::atomic<int> cache[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 1;
    if (dev < kMaxDevices) {
        const int c = cache[dev].load(std::memory_order_relaxed);
        if (c > 0) return c;
    }
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 1;
    if (dev < kMaxDevices) cache[dev].store(n, std::memory_order_relaxed);
    return n;
}

cudaError_t ensure_smem(const void *kernel, int bytes) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(g_attr_mutex);
    int &cached = g_smem_attr[std::make_pair(kernel, dev)];
    if (cached >= bytes) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) cached = bytes;
    return e;
}

}  // namespace precog

namespace {

precog_status encode_chunks(const precog_scan_inputs *in, const int64_t *d_offsets, int64_t n_chunks,
                            int64_t T_tot, void *states_out, int32_t state_dtype, int32_t layer0,
                            int32_t L_total, void *y_out, int32_t y_dtype, const int64_t *d_order,
                            void *stream) {
    if (T_tot < 0) return fail(PRECOG_ERR_INVALID_ARG, "T_tot must be >= 0");
    precog_status s = check_scan_inputs(in, T_tot, y_out != nullptr);
    if (s != PRECOG_OK) return s;
    if (n_chunks < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_chunks must be >= 0");
    if (d_offsets == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "d_offsets is NULL");
    if (states_out == nullptr && y_out == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "states_out and y_out are both NULL: nothing to do");
    if (states_out) {
        if (!state_dtype_ok(state_dtype))
            return fail(PRECOG_ERR_UNSUPPORTED, "state_dtype must be PRECOG_F32 or PRECOG_BF16");
        if (!aligned16(states_out)) return fail(PRECOG_ERR_INVALID_ARG, "states_out not 16-byte aligned");
        if (layer0 < 0 || L_total < 1 || layer0 + in->n_layers > L_total)
            return fail(PRECOG_ERR_INVALID_ARG, "layers [layer0, layer0+n_layers) exceed L_total");
    }
    if (y_out) {
        if (!state_dtype_ok(y_dtype))
            return fail(PRECOG_ERR_UNSUPPORTED, "y_dtype must be PRECOG_F32 or PRECOG_BF16");
        if (!aligned16(y_out)) return fail(PRECOG_ERR_INVALID_ARG, "y_out not 16-byte aligned");
    }
    if (n_chunks == 0) return ok();
    precog::ScanParams p = base_params(in, T_tot);
    p.offsets = d_offsets;
    p.order = d_order;
    p.n_chunks = n_chunks;
    p.states = states_out;
    p.state_dtype = state_dtype;
    p.L_out = L_total;
    p.layer0 = states_out ? layer0 : 0;
    p.y = y_out;
    p.y_dtype = y_dtype;
    cudaError_t e = in->a_kind == PRECOG_A_COMPLEX
                        ? precog::launch_scan_complex(p, static_cast<cudaStream_t>(stream))
                        : precog::launch_scan(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "scan launch");
    return ok();
}

}  // namespace

extern "C" {

precog_status precog_encode_chunks(const precog_scan_inputs *in, const int64_t *d_offsets,
                                   int64_t n_chunks, int64_t T_tot, void *states_out,
                                   int32_t state_dtype, int32_t layer0, int32_t L_total,
                                   void *y_out, int32_t y_dtype, void *stream) {
    return encode_chunks(in, d_offsets, n_chunks, T_tot, states_out, state_dtype, layer0, L_total, y_out,
                         y_dtype, nullptr, stream);
}

precog_status precog_encode_chunks_ordered(const precog_scan_inputs *in, const int64_t *d_offsets,
                                           int64_t n_chunks, int64_t T_tot, const int64_t *d_order,
                                           void *states_out, int32_t state_dtype, int32_t layer0,
                                           int32_t L_total, void *y_out, int32_t y_dtype, void *stream) {
    if (d_order == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "d_order is NULL");
    return encode_chunks(in, d_offsets, n_chunks, T_tot, states_out, state_dtype, layer0, L_total, y_out,
                         y_dtype, d_order, stream);
}

precog_status precog_prefill_from_state(const precog_scan_inputs *in, int32_t n_queries,
                                        int32_t T_q, const void *bank, int32_t bank_dtype,
                                        int64_t bank_entries, int32_t L_bank, int32_t layer0,
                                        const int64_t *d_idx, void *y_out, int32_t y_dtype,
                                        void *state_out, int32_t state_dtype, void *stream) {
    if (n_queries < 0 || T_q < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_queries and T_q must be >= 0");
    const int64_t rows = static_cast<int64_t>(n_queries) * T_q;
    precog_status s = check_scan_inputs(in, rows, y_out != nullptr);
    if (s != PRECOG_OK) return s;
    if (bank == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "bank is NULL");
    if (!state_dtype_ok(bank_dtype))
        return fail(PRECOG_ERR_UNSUPPORTED, "bank_dtype must be PRECOG_F32 or PRECOG_BF16");
    if (!aligned16(bank)) return fail(PRECOG_ERR_INVALID_ARG, "bank not 16-byte aligned");
    if (bank_entries < 0) return fail(PRECOG_ERR_INVALID_ARG, "bank_entries must be >= 0");
    if (L_bank < 1 || layer0 < 0 || layer0 + in->n_layers > L_bank)
        return fail(PRECOG_ERR_INVALID_ARG, "layers [layer0, layer0+n_layers) exceed L_bank");
    if (d_idx == nullptr && bank_entries < n_queries)
        return fail(PRECOG_ERR_INVALID_ARG, "d_idx is NULL but bank has fewer rows than queries");
    if (y_out == nullptr && state_out == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "y_out and state_out are both NULL: nothing to do");
    if (y_out && (!state_dtype_ok(y_dtype) || !aligned16(y_out)))
        return fail(PRECOG_ERR_INVALID_ARG, "y_out must be 16-byte aligned F32 or BF16");
    if (state_out && (!state_dtype_ok(state_dtype) || !aligned16(state_out)))
        return fail(PRECOG_ERR_INVALID_ARG, "state_out must be 16-byte aligned F32 or BF16");
    if (n_queries == 0) return ok();
    precog::ScanParams p = base_params(in, rows);
    p.n_chunks = n_queries;
    p.use_fixed = 1;
    p.fixed_len = T_q;
    p.bank = bank;
    p.bank_dtype = bank_dtype;
    p.bank_entries = bank_entries;
    p.idx = d_idx;
    p.L_bank = L_bank;
    p.states = state_out;
    p.state_dtype = state_dtype;
    p.L_out = L_bank;
    p.layer0 = layer0;
    p.y = y_out;
    p.y_dtype = y_dtype;
    cudaError_t e = in->a_kind == PRECOG_A_COMPLEX
                        ? precog::launch_scan_complex(p, static_cast<cudaStream_t>(stream))
                        : precog::launch_scan(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "prefill launch");
    return ok();
}

precog_status precog_encode_trajectory(const precog_scan_inputs *in, const int64_t *d_offsets,
                                       int64_t n_chunks, int64_t T_tot, int64_t stride,
                                       const int64_t *d_entry_offsets, void *traj_out,
                                       int32_t traj_dtype, int32_t layer0, int32_t L_total,
                                       void *stream) {
    if (T_tot < 0) return fail(PRECOG_ERR_INVALID_ARG, "T_tot must be >= 0");
    precog_status s = check_scan_inputs(in, T_tot, false);
    if (s != PRECOG_OK) return s;
    if (n_chunks < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_chunks must be >= 0");
    if (stride < 1) return fail(PRECOG_ERR_INVALID_ARG, "stride must be >= 1");
    if (in->a_kind == PRECOG_A_COMPLEX)
        return fail(PRECOG_ERR_UNSUPPORTED, "trajectories of a complex-A scan are not implemented");
    if (d_offsets == nullptr || d_entry_offsets == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "d_offsets and d_entry_offsets must be non-NULL");
    if (traj_out == nullptr || !state_dtype_ok(traj_dtype) || !aligned16(traj_out))
        return fail(PRECOG_ERR_INVALID_ARG, "traj_out must be a 16-byte aligned F32 or BF16 array");
    if (layer0 < 0 || L_total < 1 || layer0 + in->n_layers > L_total)
        return fail(PRECOG_ERR_INVALID_ARG, "layers [layer0, layer0+n_layers) exceed L_total");
    if (n_chunks == 0) return ok();
    precog::ScanParams p = base_params(in, T_tot);
    p.offsets = d_offsets;
    p.n_chunks = n_chunks;
    p.L_out = L_total;
    p.layer0 = layer0;
    p.traj = traj_out;
    p.traj_dtype = traj_dtype;
    p.traj_stride = stride;
    p.traj_offsets = d_entry_offsets;
    cudaError_t e = precog::launch_scan(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "trajectory launch");
    return ok();
}

precog_status precog_prefill_composed(const precog_scan_inputs *in, int32_t n_queries, int32_t T_q,
                                     const void *bank, int32_t bank_dtype, int64_t bank_entries,
                                     int32_t L_bank, int32_t layer0, int32_t k,
                                     const int64_t *d_idx, const float *d_score, float temperature,
                                     void *y_out, int32_t y_dtype, void *state_out,
                                     int32_t state_dtype, void *stream) {
    if (k < 1 || k > 8) return fail(PRECOG_ERR_UNSUPPORTED, "k must be in [1, 8]");
    if (d_idx == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "d_idx is NULL");
    if (in != nullptr && in->a_kind == PRECOG_A_COMPLEX && k > 1)
        return fail(PRECOG_ERR_UNSUPPORTED, "composition of complex states is not implemented");
    if (k > 1 && d_score == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "d_score is NULL");
    if (!(temperature > 0.f)) return fail(PRECOG_ERR_INVALID_ARG, "temperature must be > 0");
    if (k == 1)
        return precog_prefill_from_state(in, n_queries, T_q, bank, bank_dtype, bank_entries, L_bank,
                                         layer0, d_idx, y_out, y_dtype, state_out, state_dtype, stream);
    if (n_queries < 0 || T_q < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_queries and T_q must be >= 0");
    const int64_t rows = static_cast<int64_t>(n_queries) * T_q;
    precog_status s = check_scan_inputs(in, rows, y_out != nullptr);
    if (s != PRECOG_OK) return s;
    if (bank == nullptr || !state_dtype_ok(bank_dtype) || !aligned16(bank))
        return fail(PRECOG_ERR_INVALID_ARG, "bank must be a 16-byte aligned F32 or BF16 array");
    if (bank_entries < 0) return fail(PRECOG_ERR_INVALID_ARG, "bank_entries must be >= 0");
    if (L_bank < 1 || layer0 < 0 || layer0 + in->n_layers > L_bank)
        return fail(PRECOG_ERR_INVALID_ARG, "layers [layer0, layer0+n_layers) exceed L_bank");
    if (y_out == nullptr && state_out == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "y_out and state_out are both NULL: nothing to do");
    if (y_out && (!state_dtype_ok(y_dtype) || !aligned16(y_out)))
        return fail(PRECOG_ERR_INVALID_ARG, "y_out must be 16-byte aligned F32 or BF16");
    if (state_out && (!state_dtype_ok(state_dtype) || !aligned16(state_out)))
        return fail(PRECOG_ERR_INVALID_ARG, "state_out must be 16-byte aligned F32 or BF16");
    if (n_queries == 0) return ok();
    precog::ScanParams p = base_params(in, rows);
    p.n_chunks = n_queries;
    p.use_fixed = 1;
    p.fixed_len = T_q;
    p.bank = bank;
    p.bank_dtype = bank_dtype;
    p.bank_entries = bank_entries;
    p.idx = d_idx;
    p.topk = k;
    p.topk_scores = d_score;
    p.inv_temp = 1.f / temperature;
    p.L_bank = L_bank;
    p.states = state_out;
    p.state_dtype = state_dtype;
    p.L_out = L_bank;
    p.layer0 = layer0;
    p.y = y_out;
    p.y_dtype = y_dtype;
    cudaError_t e = precog::launch_scan(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "composed prefill launch");
    return ok();
}

size_t precog_retrieve_topk_workspace_size(int64_t M, int32_t dim, int32_t n_queries) {
    if (M < 0 || dim < 1 || n_queries < 0) return 0;
    return precog::retrieve_topk_workspace_size(M, dim, n_queries);
}

precog_status precog_retrieve_topk(const void *index, int32_t index_dtype, int64_t M, int32_t dim,
                                   const void *queries, int32_t n_queries, int32_t k,
                                   int64_t *d_idx, float *d_score, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    if (k < 1 || k > 8) return fail(PRECOG_ERR_UNSUPPORTED, "k must be in [1, 8]");
    const int sz = dtype_size(index_dtype);
    if (sz == 0) return fail(PRECOG_ERR_UNSUPPORTED, "index_dtype must be F16, BF16 or F32");
    if (M < 0) return fail(PRECOG_ERR_INVALID_ARG, "M must be >= 0");
    if (M >= 0x7fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "M must be below 2^31-1");
    if (dim < 1) return fail(PRECOG_ERR_INVALID_ARG, "dim must be >= 1");
    if ((static_cast<int64_t>(dim) * sz) % 16 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "dim*sizeof(dtype) must be a multiple of 16");
    if (static_cast<int64_t>(dim) * sz > 8192)
        return fail(PRECOG_ERR_UNSUPPORTED, "rows longer than 8 KiB (dim*sizeof(dtype)) are not implemented");
    if (n_queries < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_queries must be >= 0");
    if (n_queries == 0) return ok();
    if ((M > 0 && index == nullptr) || queries == nullptr || d_idx == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "index, queries and d_idx must be non-NULL");
    if ((index && !aligned16(index)) || !aligned16(queries))
        return fail(PRECOG_ERR_INVALID_ARG, "index and queries must be 16-byte aligned");
    const size_t need = precog::retrieve_topk_workspace_size(M, dim, n_queries);
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned16(workspace))))
        return fail(PRECOG_ERR_INVALID_ARG, "workspace too small or misaligned (%zu bytes needed)", need);
    precog::RetrieveParams p;
    p.index = index;
    p.dtype = index_dtype;
    p.M = M;
    p.dim = dim;
    p.queries = queries;
    p.n_queries = n_queries;
    p.best_idx = d_idx;
    p.best_score = d_score;
    p.workspace = workspace;
    p.workspace_bytes = workspace_bytes;
    cudaError_t e = precog::launch_retrieve_topk(p, k, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "top-k retrieve launch");
    return ok();
}

size_t precog_retrieve_workspace_size(int64_t M, int32_t dim, int32_t n_queries) {
    if (M < 0 || dim < 1 || n_queries < 0) return 0;
    return precog::retrieve_workspace_size(M, dim, n_queries);
}

precog_status precog_retrieve(const void *index, int32_t index_dtype, int64_t M, int32_t dim,
                              const void *queries, int32_t n_queries, int64_t *d_best_idx,
                              float *d_best_score, void *workspace, size_t workspace_bytes,
                              void *stream) {
    const int sz = dtype_size(index_dtype);
    if (sz == 0) return fail(PRECOG_ERR_UNSUPPORTED, "index_dtype must be F16, BF16 or F32");
    if (M < 0) return fail(PRECOG_ERR_INVALID_ARG, "M must be >= 0");
    if (M >= 0x7fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "M must be below 2^31-1");
    if (dim < 1) return fail(PRECOG_ERR_INVALID_ARG, "dim must be >= 1");
    if ((static_cast<int64_t>(dim) * sz) % 16 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "dim*sizeof(dtype) must be a multiple of 16");
    if (static_cast<int64_t>(dim) * sz > 8192)
        return fail(PRECOG_ERR_UNSUPPORTED, "rows longer than 8 KiB (dim*sizeof(dtype)) are not implemented");
    if (n_queries < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_queries must be >= 0");
    if (n_queries == 0) return ok();
    if ((M > 0 && index == nullptr) || queries == nullptr || d_best_idx == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "index, queries and d_best_idx must be non-NULL");
    if ((index && !aligned16(index)) || !aligned16(queries))
        return fail(PRECOG_ERR_INVALID_ARG, "index and queries must be 16-byte aligned");
    const size_t need = precog::retrieve_workspace_size(M, dim, n_queries);
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned16(workspace))))
        return fail(PRECOG_ERR_INVALID_ARG, "workspace too small or misaligned (%zu bytes needed)", need);
    precog::RetrieveParams p;
    p.index = index;
    p.dtype = index_dtype;
    p.M = M;
    p.dim = dim;
    p.queries = queries;
    p.n_queries = n_queries;
    p.best_idx = d_best_idx;
    p.best_score = d_best_score;
    p.workspace = workspace;
    p.workspace_bytes = workspace_bytes;
    cudaError_t e = precog::launch_retrieve(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "retrieve launch");
    return ok();
}

precog_status precog_retrieve_keys(const void *index, int32_t index_dtype, int64_t M, int32_t dim,
                                   const void *queries, int32_t n_queries, int64_t row_offset,
                                   int64_t *d_keys, void *workspace, size_t workspace_bytes,
                                   void *stream) {
    const int sz = dtype_size(index_dtype);
    if (sz == 0) return fail(PRECOG_ERR_UNSUPPORTED, "index_dtype must be F16, BF16 or F32");
    if (M < 0) return fail(PRECOG_ERR_INVALID_ARG, "M must be >= 0");
    if (M >= 0x7fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "M must be below 2^31-1");
    if (row_offset < 0 || row_offset + M > 0xffffffffLL)
        return fail(PRECOG_ERR_INVALID_ARG, "need row_offset >= 0 and row_offset + M <= 2^32 - 1");
    if (dim < 1) return fail(PRECOG_ERR_INVALID_ARG, "dim must be >= 1");
    if ((static_cast<int64_t>(dim) * sz) % 16 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "dim*sizeof(dtype) must be a multiple of 16");
    if (static_cast<int64_t>(dim) * sz > 8192)
        return fail(PRECOG_ERR_UNSUPPORTED, "rows longer than 8 KiB (dim*sizeof(dtype)) are not implemented");
    if (n_queries < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_queries must be >= 0");
    if (n_queries == 0) return ok();
    if ((M > 0 && index == nullptr) || queries == nullptr || d_keys == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "index, queries and d_keys must be non-NULL");
    if ((index && !aligned16(index)) || !aligned16(queries))
        return fail(PRECOG_ERR_INVALID_ARG, "index and queries must be 16-byte aligned");
    const size_t need = precog::retrieve_workspace_size(M, dim, n_queries);
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned16(workspace))))
        return fail(PRECOG_ERR_INVALID_ARG, "workspace too small or misaligned (%zu bytes needed)", need);
    precog::RetrieveParams p;
    p.index = index;
    p.dtype = index_dtype;
    p.M = M;
    p.dim = dim;
    p.queries = queries;
    p.n_queries = n_queries;
    p.best_idx = nullptr;
    p.best_score = nullptr;
    p.workspace = workspace;
    p.workspace_bytes = workspace_bytes;
    p.row_offset = row_offset;
    p.keys_out = d_keys;
    cudaError_t e = precog::launch_retrieve(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "retrieve launch");
    return ok();
}

precog_status precog_decode_keys(const int64_t *d_keys, int32_t n_queries, int64_t *d_best_idx,
                                 float *d_best_score, void *stream) {
    if (n_queries < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_queries must be >= 0");
    if (n_queries == 0) return ok();
    if (d_keys == nullptr || d_best_idx == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "d_keys and d_best_idx must be non-NULL");
    cudaError_t e = precog::launch_decode_keys(d_keys, n_queries, d_best_idx, d_best_score,
                                               static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "decode launch");
    return ok();
}

precog_status precog_smc_route(const void *embeddings, int32_t dtype, int64_t n, int32_t dim,
                               const void *domain_protos, int32_t M, const void *sub_protos,
                               int32_t J_max, const int32_t *d_J, int32_t *d_domain, int32_t *d_sub,
                               int64_t *d_slot, void *stream) {
    if (dtype_size(dtype) == 0) return fail(PRECOG_ERR_UNSUPPORTED, "dtype must be F16, BF16 or F32");
    if (n < 0 || dim < 1 || M < 0 || J_max < 0)
        return fail(PRECOG_ERR_INVALID_ARG, "n, M, J_max must be >= 0 and dim >= 1");
    if (n == 0) return ok();
    if (n > 0x7fffffffLL * 8) return fail(PRECOG_ERR_UNSUPPORTED, "too many embeddings");
    if (embeddings == nullptr || d_domain == nullptr || d_sub == nullptr ||
        (M > 0 && (domain_protos == nullptr || d_J == nullptr)) ||
        (M > 0 && J_max > 0 && sub_protos == nullptr))
        return fail(PRECOG_ERR_INVALID_ARG, "a required pointer is NULL");
    cudaError_t e = precog::launch_smc_route(embeddings, dtype, n, dim, domain_protos, M, sub_protos,
                                             J_max, d_J, d_domain, d_sub, d_slot,
                                             static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "smc route launch");
    return ok();
}

precog_status precog_smc_consolidate(float *semantic, int64_t n_slots, int64_t state_elems,
                                     const void *states, int32_t states_dtype, const int64_t *d_slots,
                                     int64_t n, float alpha, void *stream) {
    if (!state_dtype_ok(states_dtype)) return fail(PRECOG_ERR_UNSUPPORTED, "states_dtype must be F32 or BF16");
    if (n_slots < 0 || state_elems < 0 || n < 0)
        return fail(PRECOG_ERR_INVALID_ARG, "sizes must be >= 0");
    if (!(alpha > 0.f && alpha <= 1.f)) return fail(PRECOG_ERR_INVALID_ARG, "alpha must be in (0, 1]");
    if (n == 0 || state_elems == 0) return ok();
    if (semantic == nullptr || states == nullptr || d_slots == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "semantic, states and d_slots must be non-NULL");
    if (!aligned16(semantic) || !aligned16(states))
        return fail(PRECOG_ERR_INVALID_ARG, "semantic and states must be 16-byte aligned");
    cudaError_t e = precog::launch_smc_consolidate(semantic, n_slots, state_elems, states, states_dtype,
                                                   d_slots, n, alpha, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "smc consolidate launch");
    return ok();
}

precog_status precog_delta_scan(const precog_delta_inputs *in, const int64_t *d_offsets, int64_t n_seqs,
                                int64_t T_tot, const void *bank, int32_t bank_dtype, int64_t bank_entries,
                                const int64_t *d_idx, void *states_out, int32_t state_dtype, int32_t layer,
                                int32_t L_total, void *y_out, int32_t y_dtype, void *workspace,
                                size_t workspace_bytes, void *stream) {
    if (T_tot < 0) return fail(PRECOG_ERR_INVALID_ARG, "T_tot must be >= 0");
    if (T_tot >= 0x7fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "T_tot must be below 2^31-1");
    precog_status s = check_delta_inputs(in, T_tot, y_out != nullptr);
    if (s != PRECOG_OK) return s;
    if (n_seqs < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_seqs must be >= 0");
    if (d_offsets == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "d_offsets is NULL");
    if (states_out == nullptr && y_out == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "states_out and y_out are both NULL: nothing to do");
    if ((bank || states_out) && (L_total < 1 || layer < 0 || layer >= L_total))
        return fail(PRECOG_ERR_INVALID_ARG, "layer must be in [0, L_total)");
    if (bank) {
        if (!state_dtype_ok(bank_dtype))
            return fail(PRECOG_ERR_UNSUPPORTED, "bank_dtype must be PRECOG_F32 or PRECOG_BF16");
        if (!aligned16(bank)) return fail(PRECOG_ERR_INVALID_ARG, "bank not 16-byte aligned");
        if (bank_entries < 0) return fail(PRECOG_ERR_INVALID_ARG, "bank_entries must be >= 0");
        if (d_idx == nullptr && bank_entries < n_seqs)
            return fail(PRECOG_ERR_INVALID_ARG, "d_idx is NULL but bank has fewer rows than sequences");
    } else if (d_idx) {
        return fail(PRECOG_ERR_INVALID_ARG, "d_idx is given without a bank");
    }
    if (states_out && (!state_dtype_ok(state_dtype) || !aligned16(states_out)))
        return fail(PRECOG_ERR_INVALID_ARG, "states_out must be 16-byte aligned F32 or BF16");
    if (y_out && (!state_dtype_ok(y_dtype) || !aligned16(y_out)))
        return fail(PRECOG_ERR_INVALID_ARG, "y_out must be 16-byte aligned F32 or BF16");
    if (n_seqs == 0) return ok();
    if (n_seqs > kMaxItems / in->n_v_heads / ((in->dv + 15) / 16))
        return fail(PRECOG_ERR_UNSUPPORTED, "too many sequences for one call");
    precog::DeltaParams p = delta_params(in);
    p.offsets = d_offsets;
    p.n_seqs = n_seqs;
    p.T_tot = T_tot;
    const size_t need = precog::delta_scan_workspace_size(p);
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned16(workspace))))
        return fail(PRECOG_ERR_INVALID_ARG, "workspace too small or misaligned (%zu bytes needed)", need);
    p.bank = bank;
    p.bank_dtype = bank_dtype;
    p.bank_entries = bank_entries;
    p.idx = d_idx;
    p.states = states_out;
    p.state_dtype = state_dtype;
    p.layer = layer;
    p.L_total = L_total;
    p.y = y_out;
    p.y_dtype = y_dtype;
    p.workspace = workspace;
    cudaError_t e = precog::launch_delta_scan(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "delta scan launch");
    return ok();
}

size_t precog_delta_scan_workspace_size(const precog_delta_inputs *in, int64_t n_seqs, int64_t T_tot) {
    if (T_tot < 0 || T_tot >= 0x7fffffffLL || n_seqs < 1 || check_delta_inputs(in, 0, false) != PRECOG_OK) return 0;
    precog::DeltaParams p = delta_params(in);
    p.n_seqs = n_seqs;
    p.T_tot = T_tot;
    return precog::delta_scan_workspace_size(p);
}

precog_status precog_delta_step(const precog_delta_inputs *in, int64_t n, float *states, int64_t n_slots,
                                const int64_t *d_slots, int32_t layer, int32_t L_total, void *y_out,
                                int32_t y_dtype, void *stream) {
    if (n < 0) return fail(PRECOG_ERR_INVALID_ARG, "n must be >= 0");
    precog_status s = check_delta_inputs(in, n, true);
    if (s != PRECOG_OK) return s;
    if (states == nullptr || !aligned16(states))
        return fail(PRECOG_ERR_INVALID_ARG, "states must be non-NULL and 16-byte aligned");
    if (L_total < 1 || layer < 0 || layer >= L_total)
        return fail(PRECOG_ERR_INVALID_ARG, "layer must be in [0, L_total)");
    if (n_slots < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_slots must be >= 0");
    if (d_slots == nullptr && n_slots < n)
        return fail(PRECOG_ERR_INVALID_ARG, "d_slots is NULL but the table has fewer slots than rows");
    if (y_out == nullptr || !state_dtype_ok(y_dtype) || !aligned16(y_out))
        return fail(PRECOG_ERR_INVALID_ARG, "y_out must be 16-byte aligned F32 or BF16");
    if (n == 0) return ok();
    if (n > kMaxItems / in->n_v_heads / ((in->dv + 15) / 16))
        return fail(PRECOG_ERR_UNSUPPORTED, "too many rows for one call");
    precog::DeltaParams p = delta_params(in);
    p.n_seqs = n;
    p.T_tot = n;
    p.bank_entries = n_slots;
    p.idx = d_slots;
    p.states = states;
    p.state_dtype = PRECOG_F32;
    p.layer = layer;
    p.L_total = L_total;
    p.y = y_out;
    p.y_dtype = y_dtype;
    cudaError_t e = precog::launch_delta_step(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "delta step launch");
    return ok();
}

precog_status precog_qk_norm_rope(const precog_qk_norm_args *a, int64_t T, void *stream) {
    if (a == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "arguments pointer is NULL");
    if (T < 0) return fail(PRECOG_ERR_INVALID_ARG, "T must be >= 0");
    const int sz = dtype_size(a->dtype);
    if (sz == 0) return fail(PRECOG_ERR_UNSUPPORTED, "dtype must be F16, BF16 or F32");
    if (a->n_q_heads < 0 || a->n_k_heads < 0) return fail(PRECOG_ERR_INVALID_ARG, "numbers of heads must be >= 0");
    if (a->dim < 8 || a->dim > 256 || a->dim % 8 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "dim=%d: a multiple of 8 in [8, 256] is implemented", a->dim);
    if (a->n_q_heads > 0x7fffffff / a->dim || a->n_k_heads > 0x7fffffff / a->dim)
        return fail(PRECOG_ERR_UNSUPPORTED, "rows of 2^31 entries or more are not implemented");
    if (a->rot_dim < 0 || a->rot_dim > a->dim || a->rot_dim % 2 != 0)
        return fail(PRECOG_ERR_INVALID_ARG, "rot_dim must be even and in [0, dim]");
    if (a->norm < PRECOG_NORM_NONE || a->norm > PRECOG_NORM_RMS)
        return fail(PRECOG_ERR_INVALID_ARG, "norm must be PRECOG_NORM_NONE, _L2 or _RMS");
    if (a->interleaved != 0 && a->interleaved != 1) return fail(PRECOG_ERR_INVALID_ARG, "interleaved must be 0 or 1");
    if (!(a->eps >= 0.f)) return fail(PRECOG_ERR_INVALID_ARG, "eps must be >= 0");
    if (a->rot_dim > 0) {
        if (a->cos == nullptr || a->sin == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "rot_dim > 0 needs cos and sin");
        if ((reinterpret_cast<uintptr_t>(a->cos) | reinterpret_cast<uintptr_t>(a->sin)) & 3u)
            return fail(PRECOG_ERR_INVALID_ARG, "cos and sin must be 4-byte aligned");
        if (a->n_positions < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_positions must be >= 0");
        if (a->d_positions == nullptr && a->n_positions < T)
            return fail(PRECOG_ERR_INVALID_ARG, "d_positions is NULL but the tables have fewer rows than tokens");
    }
    precog::QkNormParams p;
    p.in[0] = a->q, p.in[1] = a->k;
    p.out[0] = a->q_out, p.out[1] = a->k_out;
    p.in_stride[0] = a->q_stride, p.in_stride[1] = a->k_stride;
    p.out_stride[0] = a->q_out_stride, p.out_stride[1] = a->k_out_stride;
    p.weight[0] = a->q_weight, p.weight[1] = a->k_weight;
    p.heads[0] = a->n_q_heads, p.heads[1] = a->n_k_heads;
    for (int i = 0; i < 2; ++i) {
        if (p.heads[i] == 0 || T == 0) continue;
        if (p.in[i] == nullptr || p.out[i] == nullptr)
            return fail(PRECOG_ERR_INVALID_ARG, "q, k, q_out and k_out must be non-NULL where there are heads");
        if (!aligned16(p.in[i]) || !aligned16(p.out[i]) || !aligned16(p.weight[i]))
            return fail(PRECOG_ERR_INVALID_ARG, "q, k, their outputs and weights must be 16-byte aligned");
        if (T > 1) {
            const int64_t row = static_cast<int64_t>(p.heads[i]) * a->dim;
            if (p.in_stride[i] < row || p.out_stride[i] < row)
                return fail(PRECOG_ERR_INVALID_ARG, "row strides smaller than a row");
            if ((p.in_stride[i] * sz) % 16 != 0 || (p.out_stride[i] * sz) % 16 != 0)
                return fail(PRECOG_ERR_INVALID_ARG, "row strides must keep 16-byte alignment");
        } else {
            p.in_stride[i] = p.out_stride[i] = 0;
        }
    }
    if (T == 0 || p.heads[0] + static_cast<int64_t>(p.heads[1]) == 0) return ok();
    if (T > 0x7fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "T must be below 2^31");
    p.dim = a->dim;
    p.rot = a->rot_dim;
    p.dtype = a->dtype;
    p.norm = a->norm;
    p.interleaved = a->interleaved;
    p.eps = a->eps;
    p.cos = a->cos;
    p.sin = a->sin;
    p.n_positions = a->n_positions;
    p.positions = a->d_positions;
    p.T = T;
    cudaError_t e = precog::launch_qk_norm(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "qk norm launch");
    return ok();
}

precog_status precog_token_logprobs(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab,
                                    int64_t row_stride, const int64_t *d_tokens, float temperature, int32_t k,
                                    float *d_logprob, float *d_entropy, int64_t *d_top_idx,
                                    float *d_top_logprob, void *stream) {
    const int sz = dtype_size(dtype);
    if (sz == 0) return fail(PRECOG_ERR_UNSUPPORTED, "dtype must be F16, BF16 or F32");
    if (n_rows < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_rows must be >= 0");
    if (vocab < 1) return fail(PRECOG_ERR_INVALID_ARG, "vocab must be >= 1");
    if (vocab > 0x3fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "vocab must be below 2^30");
    if (row_stride < vocab && n_rows > 1) return fail(PRECOG_ERR_INVALID_ARG, "row_stride must be >= vocab");
    if (!(temperature > 0.f) || !(1.f / temperature > 0.f) || !(1.f / temperature * 1.442695f < 3.4e38f))
        return fail(PRECOG_ERR_INVALID_ARG, "temperature and log2(e) / temperature must be positive and finite");
    if (k < 0 || k > 32) return fail(PRECOG_ERR_UNSUPPORTED, "k must be in [0, 32]");
    if (k > vocab) return fail(PRECOG_ERR_INVALID_ARG, "k must be at most vocab");
    if (n_rows == 0) return ok();
    if (logits == nullptr || d_tokens == nullptr || d_logprob == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "logits, d_tokens and d_logprob must be non-NULL");
    if (k > 0 && (d_top_idx == nullptr || d_top_logprob == nullptr))
        return fail(PRECOG_ERR_INVALID_ARG, "k > 0 needs d_top_idx and d_top_logprob");
    if ((reinterpret_cast<uintptr_t>(logits) & static_cast<uintptr_t>(sz - 1)) != 0)
        return fail(PRECOG_ERR_INVALID_ARG, "logits must be aligned to their elements");
    if (n_rows > 0x7fffffffLL / 16) return fail(PRECOG_ERR_UNSUPPORTED, "too many rows for one call");
    precog::LogprobParams p;
    p.logits = logits;
    p.dtype = dtype;
    p.rows = n_rows;
    p.vocab = vocab;
    p.stride = row_stride;
    p.tokens = d_tokens;
    p.inv_temp = 1.f / temperature;
    p.k = k;
    p.logprob = d_logprob;
    p.entropy = d_entropy;
    p.top_idx = d_top_idx;
    p.top_logprob = d_top_logprob;
    cudaError_t e = precog::launch_logprobs(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "logprobs launch");
    return ok();
}

precog_status precog_selftest_wait_timeout(uint32_t iterations, void *stream) {
    if (iterations < 1 || iterations > (1u << 20))
        return fail(PRECOG_ERR_INVALID_ARG, "iterations must be in [1, 2^20]");
    cudaError_t e = precog::launch_wait_timeout(iterations, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "self-test launch");
    return ok();
}

precog_status precog_device_status(void *stream, uint32_t *bits_out) {
    if (bits_out == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "bits_out is NULL");
    *bits_out = 0;
    cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "stream synchronize");
    StatusWords words = {};
    for (int i = 0; i < kStatusWords; ++i) {
        e = kStatusWord[i](&words.word[i]);
        if (e != cudaSuccess) return cuda_fail(e, "status word");
    }
    std::lock_guard<std::mutex> one(g_status_mutex);
    take_status_kernel<<<1, 32>>>(words);
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e, "status launch");
    e = cudaMemcpyFromSymbol(bits_out, g_taken_status, sizeof(uint32_t));
    if (e != cudaSuccess) return cuda_fail(e, "read status");
    if (*bits_out == 0) return ok();
    if (*bits_out & PRECOG_DEV_TIMEOUT)
        return fail(PRECOG_ERR_TIMEOUT, "a device-side wait gave up (bits 0x%x)", *bits_out);
    return fail(PRECOG_ERR_DEVICE, "device flagged invalid offsets, bank rows, indices or A (bits 0x%x)", *bits_out);
}

const char *precog_status_string(int32_t status) {
    switch (status) {
        case PRECOG_OK: return "PRECOG_OK";
        case PRECOG_ERR_INVALID_ARG: return "PRECOG_ERR_INVALID_ARG";
        case PRECOG_ERR_UNSUPPORTED: return "PRECOG_ERR_UNSUPPORTED";
        case PRECOG_ERR_CUDA: return "PRECOG_ERR_CUDA";
        case PRECOG_ERR_TIMEOUT: return "PRECOG_ERR_TIMEOUT";
        case PRECOG_ERR_DEVICE: return "PRECOG_ERR_DEVICE";
        default: return "PRECOG_UNKNOWN_STATUS";
    }
}

const char *precog_last_error(void) { return g_last_error; }

int32_t precog_abi_version(void) { return PRECOG_ABI_VERSION; }

uint64_t precog_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

}  // extern "C"

// ---------------------------------------------------------------------------
// Retrieval without a caller workspace.
//
// Some callers cannot allocate device memory at the moment they retrieve: a
// real-time serving loop that must not call cudaMalloc (it can synchronise the
// device and stall every stream), code running inside a memory pool owned by
// someone else, or a host whose allocator is not the CUDA one. For them the
// partial (score, row) keys of precog_retrieve live in a fixed array compiled
// into this library instead of a workspace they would have to provide.
namespace {

// 262,144 packed keys = 2 MiB, held on every GPU that loads this library until
// the process exits. Enough for about 430 queries per call at any index size on
// a 152-SM GPU (keys needed = scratch partitions x n_queries).
constexpr size_t kNoallocKeys = 262144;
static __device__ __align__(256) unsigned long long g_noalloc_scratch[kNoallocKeys];

// The array's device address belongs to one CUDA context: after cudaDeviceReset, or
// when a caller makes another context of the same device current, it is another
// address. So the address is looked up once per context (keyed by the driver's unique
// context id), not once per device number.
using CtxGetCurrentFn = CUresult (*)(CUcontext *);
using CtxGetIdFn = CUresult (*)(CUcontext, unsigned long long *);

template <typename F>
F driver_fn(const char *name) {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion(name, &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
        return reinterpret_cast<F>(p);
    return nullptr;
}

// Unique id of the calling thread's current context; false if there is none yet or the
// driver cannot tell.
bool current_context_id(unsigned long long *id) {
    static const CtxGetCurrentFn get_current = driver_fn<CtxGetCurrentFn>("cuCtxGetCurrent");
    static const CtxGetIdFn get_id = driver_fn<CtxGetIdFn>("cuCtxGetId");
    if (get_current == nullptr || get_id == nullptr) return false;
    CUcontext ctx = nullptr;
    if (get_current(&ctx) != CUDA_SUCCESS || ctx == nullptr) return false;
    return get_id(ctx, id) == CUDA_SUCCESS;
}

struct NoallocSlot {
    unsigned long long ctx_id;
    void *ptr;
};
constexpr int kNoallocSlots = 64;
std::mutex g_noalloc_mutex;
NoallocSlot g_noalloc_slots[kNoallocSlots];
int g_noalloc_filled = 0, g_noalloc_next = 0;

// Device address of the scratch in the current context. The first call in a context
// asks the runtime (cudaGetSymbolAddress, a host-side lookup that allocates nothing);
// later calls in that context reuse the answer. Without context ids every call asks.
precog_status noalloc_scratch(void **ptr) {
    unsigned long long id = 0;
    bool have_id = current_context_id(&id);
    if (have_id) {
        std::lock_guard<std::mutex> lock(g_noalloc_mutex);
        for (int i = 0; i < g_noalloc_filled; ++i)
            if (g_noalloc_slots[i].ctx_id == id) {
                *ptr = g_noalloc_slots[i].ptr;
                return PRECOG_OK;
            }
    }
    void *p = nullptr;
    const cudaError_t e = cudaGetSymbolAddress(&p, g_noalloc_scratch);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetSymbolAddress(scratch)");
    if (!have_id) have_id = current_context_id(&id);   // the lookup may have created the context
    if (have_id) {
        std::lock_guard<std::mutex> lock(g_noalloc_mutex);
        g_noalloc_slots[g_noalloc_next] = NoallocSlot{id, p};
        g_noalloc_next = (g_noalloc_next + 1) % kNoallocSlots;
        if (g_noalloc_filled < kNoallocSlots) ++g_noalloc_filled;
    }
    *ptr = p;
    return PRECOG_OK;
}

}  // namespace

extern "C" {

precog_status precog_retrieve_noalloc(const void *index, int32_t index_dtype, int64_t M,
                                      int32_t dim, const void *queries, int32_t n_queries,
                                      int64_t *d_best_idx, float *d_best_score, void *stream) {
    if (n_queries < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_queries must be >= 0");
    if (M < 0 || dim < 1) return fail(PRECOG_ERR_INVALID_ARG, "M must be >= 0 and dim >= 1");
    const size_t need = precog::retrieve_workspace_size(M, dim, n_queries);
    if (need > sizeof(g_noalloc_scratch))
        return fail(PRECOG_ERR_UNSUPPORTED,
                    "precog_retrieve_noalloc: %d queries need %zu bytes of scratch, more than the "
                    "fixed %zu; use fewer queries per call or precog_retrieve with a workspace",
                    n_queries, need, sizeof(g_noalloc_scratch));
    void *scratch = nullptr;
    precog_status s = noalloc_scratch(&scratch);
    if (s != PRECOG_OK) return s;
    return precog_retrieve(index, index_dtype, M, dim, queries, n_queries, d_best_idx,
                           d_best_score, scratch, sizeof(g_noalloc_scratch), stream);
}

}  // extern "C"
