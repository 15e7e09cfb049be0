// C ABI of the PRECOG hot path: argument validation, dispatch to the
// kernels, status codes. Nothing here allocates device memory.
#include <atomic>
#include <cstdarg>
#include <initializer_list>
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

// Whether lists of 4- or 8-byte entries are aligned to them.
bool aligned_to(unsigned bytes, std::initializer_list<const void *> lists) {
    for (const void *p : lists)
        if (reinterpret_cast<uintptr_t>(p) % bytes != 0) return false;
    return true;
}

// Rows of `row` bytes, `stride` bytes apart.
struct RowSpan {
    const void *at;
    int64_t stride, row;
};

// Whether two tensors of n rows share memory. Rows of one stride may lie between one another (slices of one
// buffer); otherwise their ranges have to be apart. `same_ok`: the very same rows do not count.
bool overlap(const RowSpan &a, const RowSpan &b, int64_t n, bool same_ok) {
    if (a.at == nullptr || b.at == nullptr || n == 0 || a.row == 0 || b.row == 0) return false;
    if (same_ok && a.at == b.at && a.row == b.row && (n == 1 || a.stride == b.stride)) return false;
    using wide = __int128;   // (strides are the caller's, and may be anything)
    const wide pa = static_cast<wide>(reinterpret_cast<uintptr_t>(a.at)), pb = static_cast<wide>(reinterpret_cast<uintptr_t>(b.at));
    if (pa + static_cast<wide>(n - 1) * a.stride + a.row <= pb || pb + static_cast<wide>(n - 1) * b.stride + b.row <= pa) return false;
    if (n == 1 || a.stride != b.stride || a.stride == 0) return true;
    wide gap = (pb - pa) % a.stride;
    if (gap < 0) gap += a.stride;
    return gap < a.row || gap + b.row > a.stride;
}

// Bytes of a table [entries][layers][row bytes], as one row; false beyond 2^63.
bool table_span(const void *at, int64_t entries, int64_t layers, int64_t row, RowSpan *span) {
    const __int128 bytes = static_cast<__int128>(entries) * layers;
    if (bytes > INT64_MAX || bytes * row > INT64_MAX) return false;
    *span = RowSpan{at, 0, at == nullptr ? 0 : static_cast<int64_t>(bytes * row)};
    return true;
}

// The range of all of a tensor's rows, as one row.
RowSpan whole(const RowSpan &a, int64_t n) {
    if (a.at == nullptr || n == 0) return RowSpan{a.at, 0, 0};
    const __int128 bytes = static_cast<__int128>(n - 1) * a.stride + a.row;
    return RowSpan{a.at, 0, bytes > INT64_MAX ? INT64_MAX : static_cast<int64_t>(bytes)};
}

// Whether one of n rows shares memory with `bytes` at `at`. What lies between strided rows is nobody's.
bool touches(const RowSpan &a, int64_t n, const void *at, __int128 bytes) {
    if (a.at == nullptr || at == nullptr || n == 0 || a.row == 0 || bytes <= 0) return false;
    using wide = __int128;
    const wide pa = static_cast<wide>(reinterpret_cast<uintptr_t>(a.at)), pb = static_cast<wide>(reinterpret_cast<uintptr_t>(at));
    if (pb + bytes <= pa || pb >= pa + static_cast<wide>(n - 1) * a.stride + a.row) return false;   // (as a rule)
    wide i = 0;   // the first row that ends behind `at`
    if (n > 1 && a.stride > 0 && pb - pa >= a.row) i = (pb - pa - a.row) / a.stride + 1;
    return i < n && pa + i * a.stride + a.row > pb && pa + i * a.stride < pb + bytes;
}

// The same of several lists (what is not given is nullptr).
struct List {
    const void *at;
    __int128 bytes;
};
bool touches_any(const RowSpan &a, int64_t n, std::initializer_list<List> lists) {
    for (const List &list : lists)
        if (touches(a, n, list.at, list.bytes)) return true;
    return false;
}

// Checks shared by the convolution's two calls; fills what they have in common.
precog_status check_conv(const precog_conv_args *a, int64_t rows, int32_t layer, int32_t L_total, precog::ConvParams *p) {
    if (a == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "arguments pointer is NULL");
    if (a->dtype != PRECOG_F32 && a->dtype != PRECOG_BF16)
        return fail(PRECOG_ERR_UNSUPPORTED, "dtype must be PRECOG_F32 or PRECOG_BF16");
    const int sz = dtype_size(a->dtype);
    if (a->dim < 8 || a->dim % 8 != 0) return fail(PRECOG_ERR_UNSUPPORTED, "dim=%d: a positive multiple of 8 is implemented", a->dim);
    if (a->kernel < 2 || a->kernel > 4) return fail(PRECOG_ERR_UNSUPPORTED, "kernel=%d: 2, 3 and 4 are implemented", a->kernel);
    if (a->silu != 0 && a->silu != 1) return fail(PRECOG_ERR_INVALID_ARG, "silu must be 0 or 1");
    if (L_total < 1 || layer < 0 || layer >= L_total) return fail(PRECOG_ERR_INVALID_ARG, "layer must be in [0, L_total)");
    if (a->weight == nullptr || !aligned16(a->weight) || !aligned16(a->bias))
        return fail(PRECOG_ERR_INVALID_ARG, "weight must be non-NULL, weight and bias 16-byte aligned");
    std::memset(p, 0, sizeof(*p));
    p->x = a->x, p->y = a->y;
    p->x_stride = rows > 1 ? a->x_stride : 0, p->y_stride = rows > 1 ? a->y_stride : 0;
    if (rows > 0) {
        if (a->x == nullptr || a->y == nullptr || !aligned16(a->x) || !aligned16(a->y))
            return fail(PRECOG_ERR_INVALID_ARG, "x and y must be non-NULL and 16-byte aligned");
        if (rows > 1 && (a->x_stride < a->dim || a->y_stride < a->dim))
            return fail(PRECOG_ERR_INVALID_ARG, "row strides smaller than a row");
        if ((p->x_stride * sz) % 16 != 0 || (p->y_stride * sz) % 16 != 0)
            return fail(PRECOG_ERR_INVALID_ARG, "row strides must keep 16-byte alignment");
    }
    p->weight = a->weight, p->bias = a->bias;
    p->dim = a->dim, p->kernel = a->kernel, p->dtype = a->dtype, p->silu = a->silu;
    p->layer = layer, p->L_total = L_total;
    return PRECOG_OK;
}

// The kernel files' status words, taken and cleared at once: a copy of each would wait for the device
// every time (eleven words: 144 us a call, so 22).
constexpr cudaError_t (*kStatusWord[])(uint32_t **) = {
    precog::scan_status_word,    precog::scan_complex_status_word, precog::scan_latency_status_word, precog::retrieve_status_word,
    precog::retrieve_tc_status_word, precog::smc_status_word,      precog::selftest_status_word,     precog::delta_status_word,
    precog::delta_chunk_status_word, precog::qk_norm_status_word,  precog::logprobs_status_word,     precog::conv_status_word,
    precog::scan_step_status_word, precog::adjust_status_word};
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

precog_status precog_causal_conv(const precog_conv_args *args, const int64_t *d_offsets, int64_t n_seqs, int64_t T_tot,
                                 const void *bank, int64_t bank_entries, const int64_t *d_idx, void *windows_out,
                                 int32_t layer, int32_t L_total, void *stream) {
    if (T_tot < 0) return fail(PRECOG_ERR_INVALID_ARG, "T_tot must be >= 0");
    if (n_seqs < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_seqs must be >= 0");
    precog::ConvParams p;
    if (T_tot > 0x7fffffffLL || n_seqs > 0x3fffffffLL)
        return fail(PRECOG_ERR_UNSUPPORTED, "T_tot must be below 2^31, n_seqs below 2^30");
    precog_status s = check_conv(args, T_tot, layer, L_total, &p);
    if (s != PRECOG_OK) return s;
    if (d_offsets == nullptr || !aligned_to(8, {d_offsets, d_idx}))
        return fail(PRECOG_ERR_INVALID_ARG, "d_offsets must be non-NULL, d_offsets and d_idx 8-byte aligned");
    if (bank) {
        if (!aligned16(bank)) return fail(PRECOG_ERR_INVALID_ARG, "bank not 16-byte aligned");
        if (bank_entries < 0) return fail(PRECOG_ERR_INVALID_ARG, "bank_entries must be >= 0");
        if (d_idx == nullptr && bank_entries < n_seqs)
            return fail(PRECOG_ERR_INVALID_ARG, "d_idx is NULL but bank has fewer rows than sequences");
    } else {
        bank_entries = 0;   // (and what d_idx names has to be -1)
    }
    if (!aligned16(windows_out)) return fail(PRECOG_ERR_INVALID_ARG, "windows_out not 16-byte aligned");
    const int64_t sz = dtype_size(p.dtype), row = p.dim * sz;
    const RowSpan x{p.x, p.x_stride * sz, row}, y{p.y, p.y_stride * sz, row};
    RowSpan from, to;
    if (!table_span(bank, bank ? bank_entries : 0, L_total, row * (p.kernel - 1), &from) ||
        !table_span(windows_out, n_seqs, L_total, row * (p.kernel - 1), &to))
        return fail(PRECOG_ERR_UNSUPPORTED, "tables beyond 2^63 bytes");
    if (overlap(x, y, T_tot, false))
        return fail(PRECOG_ERR_INVALID_ARG, "y must not share memory with x: tokens read the inputs before them");
    // a sequence's window is written while other parts of it may still read theirs
    if (overlap(from, to, 1, false)) return fail(PRECOG_ERR_INVALID_ARG, "windows_out must not share memory with bank");
    if (overlap(whole(x, T_tot), to, 1, false) || overlap(whole(y, T_tot), to, 1, false) || overlap(whole(y, T_tot), from, 1, false))
        return fail(PRECOG_ERR_INVALID_ARG, "windows and rows must not share memory");
    for (const auto &[out, n] : {std::pair(y, T_tot), std::pair(to, static_cast<int64_t>(1))})
        if (touches_any(out, n, {{p.weight, 4LL * p.dim * p.kernel}, {p.bias, 4LL * p.dim}, {d_offsets, 8 * (n_seqs + 1)}, {d_idx, 8 * n_seqs}}))
            return fail(PRECOG_ERR_INVALID_ARG, "y and windows_out must not share memory with weight, bias, d_offsets or d_idx");
    if (n_seqs == 0) return ok();
    p.offsets = d_offsets;
    p.n_seqs = n_seqs;
    p.T_tot = T_tot;
    p.bank = bank;
    p.bank_entries = bank_entries;
    p.idx = d_idx;
    p.windows = windows_out;
    cudaError_t e = precog::launch_conv(p, false, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "convolution launch");
    return ok();
}

precog_status precog_conv_step(const precog_conv_args *args, int64_t n, void *windows, int64_t n_slots,
                               const int64_t *d_slots, int32_t layer, int32_t L_total, void *stream) {
    if (n < 0) return fail(PRECOG_ERR_INVALID_ARG, "n must be >= 0");
    if (n > 0x7fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "too many rows for one call");
    precog::ConvParams p;
    precog_status s = check_conv(args, n, layer, L_total, &p);
    if (s != PRECOG_OK) return s;
    if ((n > 0 && windows == nullptr) || !aligned16(windows))
        return fail(PRECOG_ERR_INVALID_ARG, "windows must be non-NULL and 16-byte aligned");
    if (n_slots < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_slots must be >= 0");
    if (!aligned_to(8, {d_slots})) return fail(PRECOG_ERR_INVALID_ARG, "d_slots not 8-byte aligned");
    if (d_slots == nullptr && n_slots < n)
        return fail(PRECOG_ERR_INVALID_ARG, "d_slots is NULL but the table has fewer slots than rows");
    const int64_t sz = dtype_size(p.dtype), row = p.dim * sz;
    const RowSpan x{p.x, p.x_stride * sz, row}, y{p.y, p.y_stride * sz, row};
    if (overlap(x, y, n, true)) return fail(PRECOG_ERR_INVALID_ARG, "y must be x itself or share no memory with it");
    RowSpan table;
    if (!table_span(windows, n_slots, L_total, row * (p.kernel - 1), &table))
        return fail(PRECOG_ERR_UNSUPPORTED, "tables beyond 2^63 bytes");
    if (overlap(whole(x, n), table, 1, false) || overlap(whole(y, n), table, 1, false))
        return fail(PRECOG_ERR_INVALID_ARG, "windows and rows must not share memory");
    for (const auto &[out, rows] : {std::pair(y, n), std::pair(table, static_cast<int64_t>(1))})
        if (touches_any(out, rows, {{p.weight, 4LL * p.dim * p.kernel}, {p.bias, 4LL * p.dim}, {d_slots, 8 * n}}))
            return fail(PRECOG_ERR_INVALID_ARG, "y and windows must not share memory with weight, bias or d_slots");
    if (n == 0) return ok();
    p.n_seqs = n;
    p.T_tot = n;
    p.bank_entries = n_slots;
    p.idx = d_slots;
    p.windows = windows;
    cudaError_t e = precog::launch_conv(p, true, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "convolution step launch");
    return ok();
}

precog_status precog_scan_step(const precog_scan_inputs *in, const precog_scan_step_args *a, int64_t n, void *stream) {
    if (a == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "arguments pointer is NULL");
    if (a->reserved != 0) return fail(PRECOG_ERR_INVALID_ARG, "reserved must be 0");
    void *const states = a->states, *const y_out = a->y_out;
    const int64_t n_slots = a->n_slots, *const d_slots = a->d_slots, gate_stride = a->gate_stride, gate_layer_stride = a->gate_layer_stride;
    const int32_t layer0 = a->layer0, L_total = a->L_total, y_dtype = a->y_dtype;
    const float *const skip = a->skip;
    const void *const gate = a->gate;
    if (n < 0) return fail(PRECOG_ERR_INVALID_ARG, "n must be >= 0");
    if (n > 0x7fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "too many rows for one call");
    precog_status s = check_scan_inputs(in, n, true);
    if (s != PRECOG_OK) return s;
    if ((n > 0 && states == nullptr) || !aligned16(states))
        return fail(PRECOG_ERR_INVALID_ARG, "states must be non-NULL and 16-byte aligned");
    if (layer0 < 0 || L_total < 1 || static_cast<int64_t>(layer0) + in->n_layers > L_total)
        return fail(PRECOG_ERR_INVALID_ARG, "layers [layer0, layer0+n_layers) exceed L_total");
    if (n_slots < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_slots must be >= 0");
    if (!aligned_to(8, {d_slots})) return fail(PRECOG_ERR_INVALID_ARG, "d_slots not 8-byte aligned");
    if (d_slots == nullptr && n_slots < n)
        return fail(PRECOG_ERR_INVALID_ARG, "d_slots is NULL but the table has fewer slots than rows");
    if ((n > 0 && y_out == nullptr) || !state_dtype_ok(y_dtype) || !aligned16(y_out))
        return fail(PRECOG_ERR_INVALID_ARG, "y_out must be 16-byte aligned F32 or BF16");
    if (!aligned16(skip) || !aligned16(gate)) return fail(PRECOG_ERR_INVALID_ARG, "skip and gate must be 16-byte aligned");
    if (gate) {
        const int sz = dtype_size(in->in_dtype);
        if ((n > 1 && gate_stride < in->D) || (in->n_layers > 1 && gate_layer_stride < in->D))
            return fail(PRECOG_ERR_INVALID_ARG, "gate strides smaller than a row");
        if ((n > 1 && (gate_stride * sz) % 16 != 0) || (in->n_layers > 1 && (gate_layer_stride * sz) % 16 != 0))
            return fail(PRECOG_ERR_INVALID_ARG, "gate strides must keep 16-byte alignment");
    }
    if (n == 0) return ok();
    const int64_t sz = dtype_size(in->in_dtype), parts = in->a_kind == PRECOG_A_COMPLEX ? 2 : 1;
    const RowSpan y{y_out, 0, in->n_layers * n * in->D * dtype_size(y_dtype)};
    const RowSpan inputs[6] = {whole(RowSpan{in->x, in->layer_stride_xd * sz, n * in->D * sz}, in->n_layers),
                               whole(RowSpan{in->dt, in->layer_stride_xd * sz, n * in->D * sz}, in->n_layers),
                               whole(RowSpan{in->B, in->layer_stride_bc * sz, n * in->N * sz}, in->n_layers),
                               whole(RowSpan{in->C, in->layer_stride_bc * sz, n * in->N * sz}, in->n_layers),
                               RowSpan{in->A, 0, 4LL * parts * in->n_layers * in->D * in->N},
                               whole(RowSpan{gate, gate_layer_stride * sz, whole(RowSpan{gate, gate_stride * sz, in->D * sz}, n).row}, in->n_layers)};
    RowSpan table;
    if (!table_span(states, n_slots, L_total, 4LL * parts * in->D * in->N, &table))
        return fail(PRECOG_ERR_UNSUPPORTED, "tables beyond 2^63 bytes");
    const int64_t skip_bytes = 4LL * in->n_layers * in->D;
    bool shared = overlap(y, table, 1, false) || touches_any(y, 1, {{skip, skip_bytes}, {d_slots, 8 * n}}) ||
                  touches_any(table, 1, {{skip, skip_bytes}, {d_slots, 8 * n}});
    for (const RowSpan &r : inputs) shared = shared || overlap(r, table, 1, false) || overlap(r, y, 1, false);
    if (shared) return fail(PRECOG_ERR_INVALID_ARG, "y_out, states and inputs must not share memory");
    precog::ScanStepParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = in->x, p.dt = in->dt, p.B = in->B, p.C = in->C, p.A = in->A;
    p.ls_xd = in->n_layers > 1 ? in->layer_stride_xd : 0;
    p.ls_bc = in->n_layers > 1 ? in->layer_stride_bc : 0;
    p.n_layers = in->n_layers, p.D = in->D, p.in_dtype = in->in_dtype;
    p.complex = in->a_kind == PRECOG_A_COMPLEX;
    p.n = n;
    p.states = static_cast<float *>(states);
    p.n_slots = n_slots;
    p.slots = d_slots;
    p.layer0 = layer0, p.L_total = L_total;
    p.skip = skip;
    p.gate = gate;
    p.gate_stride = n > 1 ? gate_stride : 0;
    p.gate_layer_stride = in->n_layers > 1 ? gate_layer_stride : 0;
    p.y = y_out, p.y_dtype = y_dtype;
    cudaError_t e = precog::launch_scan_step(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "scan step launch");
    return ok();
}

precog_status precog_block_norm(const precog_block_norm_args *a, int64_t T, void *stream) {
    if (a == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "arguments pointer is NULL");
    if (T < 0) return fail(PRECOG_ERR_INVALID_ARG, "T must be >= 0");
    if ((a->dtype != PRECOG_F32 && a->dtype != PRECOG_BF16) || (a->residual_dtype != PRECOG_F32 && a->residual_dtype != PRECOG_BF16))
        return fail(PRECOG_ERR_UNSUPPORTED, "dtype and residual_dtype must be PRECOG_F32 or PRECOG_BF16");
    if (a->residual && a->dtype == PRECOG_F32 && a->residual_dtype != PRECOG_F32)
        return fail(PRECOG_ERR_UNSUPPORTED, "a residual of F32 rows must be F32");
    if (a->groups < 1 || a->dim < 8) return fail(PRECOG_ERR_INVALID_ARG, "groups must be >= 1 and dim >= 8");
    if (a->dim % a->groups != 0 || a->dim / a->groups % 8 != 0)
        return fail(PRECOG_ERR_UNSUPPORTED, "dim / groups must be a multiple of 8");
    if (a->dim / a->groups > 16384) return fail(PRECOG_ERR_UNSUPPORTED, "norms over more than 16384 entries are not implemented");
    if (a->norm != PRECOG_NORM_NONE && a->norm != PRECOG_NORM_RMS)
        return fail(PRECOG_ERR_INVALID_ARG, "norm must be PRECOG_NORM_NONE or _RMS");
    if (a->gate_first != 0 && a->gate_first != 1) return fail(PRECOG_ERR_INVALID_ARG, "gate_first must be 0 or 1");
    if (!(a->eps >= 0.f)) return fail(PRECOG_ERR_INVALID_ARG, "eps must be >= 0");
    if (a->residual && a->out && a->groups != 1)
        return fail(PRECOG_ERR_UNSUPPORTED, "groups are not implemented with a norm of the residual");
    if (T > 0x7fffffffLL / a->groups) return fail(PRECOG_ERR_UNSUPPORTED, "too many rows for one call");
    if (T == 0) return ok();   // (rows of which there are none need no address)
    if ((a->skip == nullptr) != (a->skip_input == nullptr))
        return fail(PRECOG_ERR_INVALID_ARG, "skip and skip_input must be given together");
    if ((a->residual == nullptr) != (a->residual_out == nullptr))
        return fail(PRECOG_ERR_INVALID_ARG, "residual and residual_out must be given together");
    if (a->x == nullptr || (a->out == nullptr && a->residual_out == nullptr))
        return fail(PRECOG_ERR_INVALID_ARG, "x and one of out and residual_out must be non-NULL");
    precog::BlockNormParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = a->x, p.skip_input = a->skip_input, p.gate = a->gate, p.residual = a->residual;
    p.residual_out = a->residual_out, p.out = a->out;
    const int64_t sz = dtype_size(a->dtype), rsz = dtype_size(a->residual_dtype);
    struct {
        const void *at;
        int64_t stride, size;
        int64_t *to;
    } rows[6] = {{a->x, a->x_stride, sz, &p.x_stride},
                 {a->skip_input, a->skip_stride, sz, &p.skip_stride},
                 {a->gate, a->gate_stride, sz, &p.gate_stride},
                 {a->residual, a->residual_stride, rsz, &p.residual_stride},
                 {a->residual_out, a->residual_out_stride, rsz, &p.residual_out_stride},
                 {a->out, a->out_stride, sz, &p.out_stride}};
    RowSpan span[6];
    for (int i = 0; i < 6; ++i) {
        *rows[i].to = T > 1 ? rows[i].stride : 0;
        span[i] = RowSpan{rows[i].at, *rows[i].to * rows[i].size, a->dim * rows[i].size};
        if (rows[i].at == nullptr) continue;
        if (!aligned16(rows[i].at)) return fail(PRECOG_ERR_INVALID_ARG, "rows must be 16-byte aligned");
        if (T > 1 && rows[i].stride < a->dim) return fail(PRECOG_ERR_INVALID_ARG, "row strides smaller than a row");
        if (span[i].stride % 16 != 0) return fail(PRECOG_ERR_INVALID_ARG, "row strides must keep 16-byte alignment");
    }
    for (const float *w : {a->skip, a->weight, a->scale_weight, a->out_weight})
        for (int i = 4; i < 6; ++i)
            if (overlap(whole(span[i], T), RowSpan{w, 0, 4LL * a->dim}, 1, false))
                return fail(PRECOG_ERR_INVALID_ARG, "outputs and weights must not share memory");
    // an entry's inputs are read, by the thread that writes its outputs, before those are written
    for (int i = 0; i < 5; ++i)
        if (overlap(span[i], span[5], T, i < 4) || (i < 4 && overlap(span[i], span[4], T, true)))
            return fail(PRECOG_ERR_INVALID_ARG, "outputs must be inputs' very rows or share no memory with them or one another");
    if (!aligned16(a->skip) || !aligned16(a->weight) || !aligned16(a->scale_weight) || !aligned16(a->out_weight))
        return fail(PRECOG_ERR_INVALID_ARG, "skip and weights must be 16-byte aligned");
    p.skip = a->skip, p.weight = a->weight, p.scale_weight = a->scale_weight, p.out_weight = a->out_weight;
    p.scale = a->scale, p.eps = a->eps;
    p.dim = a->dim, p.groups = a->groups, p.dtype = a->dtype, p.residual_dtype = a->residual ? a->residual_dtype : PRECOG_F32;
    p.norm = a->norm, p.gate_first = a->gate_first;
    p.T = T;
    cudaError_t e = precog::launch_block_norm(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "block norm launch");
    return ok();
}

precog_status precog_adjust_logits(const precog_adjust_args *a, int64_t n_rows, void *stream) {
    if (a == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "arguments pointer is NULL");
    const int sz = dtype_size(a->dtype);
    if (sz == 0) return fail(PRECOG_ERR_UNSUPPORTED, "dtype must be F16, BF16 or F32");
    if (n_rows < 0) return fail(PRECOG_ERR_INVALID_ARG, "n_rows must be >= 0");
    if (a->reserved != 0) return fail(PRECOG_ERR_INVALID_ARG, "reserved must be 0");
    if (a->vocab < 1) return fail(PRECOG_ERR_INVALID_ARG, "vocab must be >= 1");
    if (a->vocab > 0x3fffffffLL) return fail(PRECOG_ERR_UNSUPPORTED, "vocab must be below 2^30");
    if (n_rows > 1 && (a->stride < a->vocab || a->out_stride < a->vocab))
        return fail(PRECOG_ERR_INVALID_ARG, "row strides must be >= vocab");
    if (a->n_history < 0 || a->n_bias < 0 || a->n_masks < 0)
        return fail(PRECOG_ERR_INVALID_ARG, "n_history, n_bias and n_masks must be >= 0");
    if (a->n_history > 0x3fffffffLL || a->n_bias > 0x3fffffffLL)
        return fail(PRECOG_ERR_UNSUPPORTED, "lists of 2^30 entries or more are not implemented");
    if (n_rows > 0x7fffffffLL / ((a->vocab + 1023) / 1024)) return fail(PRECOG_ERR_UNSUPPORTED, "too many rows for one call");
    if (n_rows == 0) return ok();
    if (a->logits == nullptr || a->out == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "logits and out must be non-NULL");
    const uintptr_t odd = static_cast<uintptr_t>(sz - 1);
    if (((reinterpret_cast<uintptr_t>(a->logits) | reinterpret_cast<uintptr_t>(a->out)) & odd) != 0)
        return fail(PRECOG_ERR_INVALID_ARG, "logits and out must be aligned to their elements");
    if (!aligned_to(8, {a->d_history, a->d_history_offsets, a->d_count_from, a->d_bias_idx, a->d_bias_offsets, a->d_mask_rows}) ||
        !aligned_to(4, {a->d_repetition, a->d_frequency, a->d_presence, a->d_bias, a->d_mask}))
        return fail(PRECOG_ERR_INVALID_ARG, "lists must be aligned to their entries");
    const bool penalised = a->d_repetition || a->d_frequency || a->d_presence;
    if (a->d_history && a->d_history_offsets == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "d_history needs d_history_offsets");
    if (a->n_history > 0 && penalised && a->d_history == nullptr)
        return fail(PRECOG_ERR_INVALID_ARG, "n_history > 0 needs d_history");
    if (a->n_bias > 0 && (a->d_bias_idx == nullptr || a->d_bias == nullptr || a->d_bias_offsets == nullptr))
        return fail(PRECOG_ERR_INVALID_ARG, "n_bias > 0 needs d_bias_idx, d_bias and d_bias_offsets");
    if (a->n_masks > 0 && a->d_mask == nullptr) return fail(PRECOG_ERR_INVALID_ARG, "n_masks > 0 needs d_mask");
    if (a->d_mask && a->d_mask_rows == nullptr && a->n_masks < n_rows)
        return fail(PRECOG_ERR_INVALID_ARG, "d_mask_rows is NULL but there are fewer masks than rows");
    precog::AdjustParams p;
    std::memset(&p, 0, sizeof(p));
    p.logits = a->logits, p.out = a->out;
    p.dtype = a->dtype;
    p.rows = n_rows, p.vocab = a->vocab;
    p.stride = n_rows > 1 ? a->stride : 0, p.out_stride = n_rows > 1 ? a->out_stride : 0;
    if (overlap(RowSpan{p.logits, p.stride * sz, p.vocab * sz}, RowSpan{p.out, p.out_stride * sz, p.vocab * sz}, n_rows, true))
        return fail(PRECOG_ERR_INVALID_ARG, "out must be logits itself or share no memory with it");
    if (a->n_history > 0 && penalised) {
        p.history = a->d_history, p.history_offsets = a->d_history_offsets, p.count_from = a->d_count_from;
        p.n_history = a->n_history;
        p.repetition = a->d_repetition, p.frequency = a->d_frequency, p.presence = a->d_presence;
    }
    if (a->n_bias > 0) p.bias_idx = a->d_bias_idx, p.bias = a->d_bias, p.bias_offsets = a->d_bias_offsets, p.n_bias = a->n_bias;
    if (a->d_mask) p.mask = reinterpret_cast<const uint32_t *>(a->d_mask), p.n_masks = a->n_masks;
    p.mask_rows = a->d_mask_rows;   // (without masks: each has to be -1)
    const int64_t per_row = 8 * n_rows, words = (p.vocab + 31) / 32;
    if (touches_any(RowSpan{p.out, p.out_stride * sz, p.vocab * sz}, n_rows,
                    {{p.history, 8 * p.n_history}, {p.history_offsets, per_row + 8}, {p.count_from, per_row}, {p.repetition, per_row / 2},
                     {p.frequency, per_row / 2}, {p.presence, per_row / 2}, {p.bias_idx, 8 * p.n_bias}, {p.bias, 4 * p.n_bias},
                     {p.bias_offsets, per_row + 8}, {p.mask, static_cast<__int128>(4 * words) * p.n_masks}, {p.mask_rows, per_row}}))
        return fail(PRECOG_ERR_INVALID_ARG, "out must not share memory with lists, vectors or masks");
    cudaError_t e = precog::launch_adjust(p, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "logit adjustment launch");
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
