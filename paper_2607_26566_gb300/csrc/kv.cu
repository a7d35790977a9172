// The host side of the key/value cache in the store's pages: the t2i_kv_* C
// ABI, its checks, and the launches.
#include <cuda.h>
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <string>

#include "common.hpp"
#include "kv.hpp"
#include "store_access.hpp"
#include "t2istore.h"

struct t2i_kv {
    t2i_store* store;
    t2i::StoreInfo info;
    t2i_kv_layout layout;
    uint32_t token_shift;
    uint32_t sms;
    uint32_t* fault;       // pinned: a kernel's wait ran out
    uint32_t* fault_dev;
    CUtensorMap map;
    uint32_t timeout_countdown;  // t2i_kv_inject_timeout
};

namespace t2i {
namespace {

constexpr uint32_t kMaxDim = 128;
constexpr uint32_t kMaxHeads = 1024;
constexpr uint32_t kMaxLayers = 1024;
constexpr uint32_t kMinPageTokens = 8;
constexpr uint64_t kMaxStride = uint64_t(1) << 40;

struct DeviceScope {
    int prev = -1;
    bool switched = false;
    explicit DeviceScope(int dev) {
        if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) switched = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceScope() {
        if (switched) cudaSetDevice(prev);
    }
};

struct Nvtx {
    explicit Nvtx(const char* name) { nvtxRangePushA(name); }
    ~Nvtx() { nvtxRangePop(); }
};

const char* layout_error(const t2i_kv_layout& l) {
    if (l.layers < 1 || l.layers > kMaxLayers) return "layers must be 1 to 1024";
    if (l.kv_heads < 1 || l.kv_heads > kMaxHeads) return "kv_heads must be 1 to 1024";
    if (l.head_dim < 8 || l.head_dim > kMaxDim || l.head_dim % 8) return "head_dim must be a multiple of 8, at most 128";
    if (l.dtype != T2I_BF16 && l.dtype != T2I_F16) return "the cache's dtype must be T2I_BF16 or T2I_F16";
    return nullptr;
}

// log2 of the tokens of a page; -1 if fewer than kMinPageTokens fit.
int page_token_shift(uint64_t page_bytes, const t2i_kv_layout& l) {
    const uint64_t token = uint64_t(l.layers) * 2 * l.kv_heads * l.head_dim * 2;
    int s = -1;
    while ((token << (s + 1)) <= page_bytes) ++s;
    return s >= 0 && (1u << s) >= kMinPageTokens ? s : -1;
}

// One call's checks. A check that fails sets the store's error; the ones after
// it do nothing.
class Checks {
  public:
    Checks(t2i_kv* kv, const char* call) : kv_(kv), call_(call) { store_check_begin(kv->store); }
    bool ok() const { return ok_; }
    void require(bool good, const char* why) {
        if (ok_ && !good) fail("", why);
    }
    // [p, p + n) is device memory, aligned
    void range(const char* name, const void* p, uint64_t n, uint32_t align) {
        if (!ok_) return;
        if (reinterpret_cast<uint64_t>(p) % align) return fail(name, ("must be " + std::to_string(align) + "-byte aligned").c_str());
        if (const char* why = store_check(kv_->store, p, n)) fail(name, why);
    }
    // [n][heads][head_dim] elements with a stride between tokens
    uint64_t token_bytes(uint64_t n, uint32_t heads, uint64_t stride, uint32_t elem) const {
        return ((n - 1) * stride + uint64_t(heads) * kv_->layout.head_dim) * elem;
    }
    void tokens(const char* name, const void* p, uint64_t n, uint32_t heads, uint64_t stride, uint32_t elem, bool written) {
        if (!ok_) return;
        if (n > 1 && (stride % 8 || stride > kMaxStride)) return fail(name, "the stride must be a multiple of 8 elements");
        if (written && n > 1 && stride < uint64_t(heads) * kv_->layout.head_dim)
            return fail(name, "the rows of an output overlap (its stride is too small)");
        range(name, p, token_bytes(n, heads, stride, elem), 16);
    }
    void table(const int32_t* t, uint64_t stride, uint32_t pages, uint32_t n_seqs) {
        require(pages > 0 && stride >= pages && stride <= kMaxStride, "table_stride must be at least table_pages, which is positive");
        // (slots are counted in 32 bits with a sign, up to the end of a tile of 128)
        require(pages <= (0x7FFFFF00u >> kv_->token_shift), "a table row must hold at most 2^31 - 256 tokens");
        if (ok_) range("table", t, ((n_seqs - 1) * stride + pages) * 4, 4);
    }
    // the batch; false (and ok()) where there is nothing to do
    bool batch(const t2i_kv_batch& b) {
        require(b.reserved == 0, "reserved must be 0");
        require(b.layer < kv_->layout.layers, "layer is not one of the layout's");
        require(b.n_tokens <= 0x7FFFFFFFu && b.n_seqs <= 0x7FFFFFFFu, "too many tokens or sequences");
        if (!ok_ || b.n_tokens == 0) return false;
        require(b.n_seqs > 0, "tokens without sequences");
        if (!ok_) return false;
        require(b.starts || b.n_tokens % b.n_seqs == 0, "without starts, n_tokens must be a multiple of n_seqs");
        table(b.table, b.table_stride, b.table_pages, b.n_seqs);
        range("lens", b.lens, uint64_t(b.n_seqs) * 4, 4);
        if (b.starts) range("starts", b.starts, (uint64_t(b.n_seqs) + 1) * 4, 4);
        return ok_;
    }
    void fail(const char* name, const char* why) {
        ok_ = false;
        store_set_error(kv_->store, std::string(call_) + ": " + name + (*name ? ": " : "") + why);
    }

  private:
    t2i_kv* kv_;
    const char* call_;
    bool ok_ = true;
};

bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    const uint64_t x = reinterpret_cast<uint64_t>(a), y = reinterpret_cast<uint64_t>(b);
    return x < y + nb && y < x + na;
}

// Whether rows of two token arrays (n rows each; bytes of a row, and from row to row) share a byte. Rows of one fused
// projection lie between one another and share none.
struct TokenRows {
    const void* p;
    uint64_t bytes, stride;
};
bool overlap(const TokenRows& a, const TokenRows& b, uint64_t n) {
    if (n > 1 && (a.stride != b.stride || !a.stride))
        return overlap(a.p, (n - 1) * a.stride + a.bytes, b.p, (n - 1) * b.stride + b.bytes);
    // row i of b lies d + (i - j) * stride behind row j of a: the first i - j that reaches into it
    const int64_t d = int64_t(reinterpret_cast<uint64_t>(b.p) - reinterpret_cast<uint64_t>(a.p));
    const int64_t s = n > 1 ? int64_t(a.stride) : 1, most = int64_t(n) - 1, past = -int64_t(b.bytes) - d;
    int64_t m = past / s - (past % s < 0 ? 1 : 0) + 1;  // (above past / s)
    if (m < -most) m = -most;
    return m <= most && d + m * s < int64_t(a.bytes);
}

KvPages pages_of(const t2i_kv* kv, const int32_t* table, uint64_t stride, uint32_t table_pages, uint32_t layer) {
    KvPages p{};
    p.pool = kv->info.pool;
    p.page_bytes = kv->info.page_bytes;
    p.total_pages = uint32_t(kv->info.total_pages);
    p.token_shift = kv->token_shift;
    p.kv_heads = kv->layout.kv_heads;
    p.head_dim = kv->layout.head_dim;
    p.layers = kv->layout.layers;
    p.layer = layer;
    p.table = table;
    p.table_stride = stride;
    p.table_pages = table_pages;
    return p;
}

KvTokens tokens_of(const t2i_kv_batch& b) {
    KvTokens t{};
    t.lens = b.lens;
    t.starts = b.starts;
    t.each = b.starts ? 0 : b.n_tokens / b.n_seqs;
    t.n_seqs = b.n_seqs;
    t.n_tokens = b.n_tokens;
    t.max_new = b.max_new ? b.max_new : t.each;
    if (t.max_new > b.n_tokens) t.max_new = b.n_tokens;
    return t;
}

template <class Launch>
t2i_status launch(t2i_kv* kv, const char* call, Launch&& go) {
    if (!store_may_launch(kv->store)) {
        store_set_error(kv->store, std::string(call) + ": kernel launch failed: injected failure (t2i_inject_launch_failure)");
        return T2I_ERR_CUDA;
    }
    DeviceScope g(kv->info.device);
    const cudaError_t e = go();
    if (e != cudaSuccess) {
        store_set_error(kv->store, std::string(call) + ": kernel launch failed: " + cudaGetErrorString(e));
        return T2I_ERR_CUDA;
    }
    store_launched(kv->store);
    return T2I_OK;
}

// Reported once, by the first call after it: what the kernel wrote is not valid.
t2i_status past_fault(t2i_kv* kv, const char* call) {
    if (*static_cast<volatile uint32_t*>(kv->fault) == 0) return T2I_OK;
    *kv->fault = 0;
    store_set_error(kv->store, std::string(call) + ": an earlier attention kernel gave up waiting for its own loads: "
                                                   "its results are not valid, and this call did nothing");
    return T2I_ERR_CUDA;
}

t2i_status append(t2i_kv* kv, const t2i_kv_append_desc& d, cudaStream_t stream) {
    Checks c(kv, "kv_append");
    const uint32_t K = kv->layout.kv_heads, D = kv->layout.head_dim;
    c.require(d.in_dtype <= T2I_F32 && d.interleaved <= 1, "in_dtype or interleaved is not one of its values");
    c.require(!d.q == !d.q_out, "q and q_out are given together or not at all");
    c.require(!d.q || (d.q_heads >= 1 && d.q_heads <= kMaxHeads), "q_heads must be 1 to 1024");
    c.require(d.rotary_dim % 2 == 0 && d.rotary_dim <= D, "rotary_dim must be even and at most head_dim");
    c.require(!d.rotary_dim || (d.n_positions > 0 && d.n_positions <= 0x7FFFFFFFu), "a rotation needs n_positions rows of its tables");
    c.require(!(d.q_norm || d.k_norm) || (std::isfinite(d.eps) && d.eps >= 0.0f), "eps must be finite and not negative");
    if (!c.batch(d.batch)) return c.ok() ? T2I_OK : T2I_ERR_INVALID;
    const t2i_status past = past_fault(kv, "kv_append");
    if (past != T2I_OK) return past;
    const uint64_t n = d.batch.n_tokens;
    const uint32_t in = d.in_dtype == T2I_F32 ? 4 : 2;
    if (d.q) {
        c.tokens("q", d.q, n, d.q_heads, d.q_stride, in, false);
        c.tokens("q_out", d.q_out, n, d.q_heads, d.q_out_stride, 2, true);
    }
    c.tokens("k", d.k, n, K, d.k_stride, in, false);
    c.tokens("v", d.v, n, K, d.v_stride, in, false);
    if (d.q_norm) c.range("q_norm", d.q_norm, D * 4, 4);
    if (d.k_norm) c.range("k_norm", d.k_norm, D * 4, 4);
    if (d.rotary_dim) {
        const uint64_t bytes = uint64_t(d.n_positions) * (d.rotary_dim / 2) * 4;
        c.range("cos_table", d.cos_table, bytes, 4);
        c.range("sin_table", d.sin_table, bytes, 4);
        if (d.positions) c.range("positions", d.positions, n * 4, 4);
    }
    if (!c.ok()) return T2I_ERR_INVALID;
    if (d.q) {
        const bool in_place = d.q == d.q_out && d.in_dtype == kv->layout.dtype && (d.q_stride == d.q_out_stride || n == 1);
        const uint64_t row = uint64_t(D) * in;
        const TokenRows to{d.q_out, uint64_t(d.q_heads) * D * 2, d.q_out_stride * 2};
        c.require(in_place || !overlap(to, {d.q, d.q_heads * row, d.q_stride * in}, n), "q_out overlaps q without being q itself");
        c.require(!overlap(to, {d.k, K * row, d.k_stride * in}, n) && !overlap(to, {d.v, K * row, d.v_stride * in}, n),
                  "q_out overlaps k or v");
        if (!c.ok()) return T2I_ERR_INVALID;
    }
    KvAppend a{};
    a.pages = pages_of(kv, d.batch.table, d.batch.table_stride, d.batch.table_pages, d.batch.layer);
    a.tok = tokens_of(d.batch);
    a.q = d.q, a.k = d.k, a.v = d.v, a.q_out = d.q_out;
    a.q_stride = d.q_stride, a.k_stride = d.k_stride, a.v_stride = d.v_stride, a.q_out_stride = d.q_out_stride;
    a.q_norm = d.q_norm, a.k_norm = d.k_norm;
    a.cos_table = d.cos_table, a.sin_table = d.sin_table;
    a.positions = d.positions;
    a.q_heads = d.q ? d.q_heads : 0;
    a.rotary_dim = d.rotary_dim;
    a.n_positions = d.n_positions;
    a.interleaved = d.interleaved;
    a.eps = d.eps;
    return launch(kv, "kv_append", [&] { return launch_kv_append(a, kv->layout.dtype, d.in_dtype, stream); });
}

uint64_t workspace_bytes(const t2i_kv* kv, uint32_t n_seqs, uint32_t n_tokens, uint32_t q_heads) {
    return std::max(kv_few_workspace(kv->sms), kv_rows_workspace(kv->sms, n_seqs, n_tokens, q_heads / kv->layout.kv_heads));
}

t2i_status attend(t2i_kv* kv, const t2i_kv_attend_desc& d, cudaStream_t stream) {
    Checks c(kv, "kv_attend");
    const uint32_t K = kv->layout.kv_heads;
    c.require(d.reserved == 0, "reserved must be 0");
    c.require(d.q_heads >= 1 && d.q_heads <= kMaxHeads && d.q_heads % K == 0, "q_heads must be a multiple of kv_heads, at most 1024");
    c.require(std::isfinite(d.scale) && std::isfinite(d.softcap) && d.softcap >= 0.0f, "scale and softcap must be finite, softcap not negative");
    c.require(!d.spans || (!d.window && !d.tree), "spans go without a window and without a tree");
    c.require(d.batch.max_new || !d.batch.starts, "with starts, max_new must be given");
    if (!c.batch(d.batch)) return c.ok() ? T2I_OK : T2I_ERR_INVALID;
    KvAttend a{};
    const t2i_status past = past_fault(kv, "kv_attend");
    if (past != T2I_OK) return past;
    a.tok = tokens_of(d.batch);
    c.require(!d.tree || a.tok.max_new <= 64, "a tree has at most 64 tokens");
    const uint64_t n = d.batch.n_tokens;
    c.tokens("q", d.q, n, d.q_heads, d.q_stride, 2, false);
    c.tokens("out", d.out, n, d.q_heads, d.out_stride, 2, true);
    if (d.lse) c.range("lse", d.lse, n * d.q_heads * 4, 4);
    if (d.slopes) c.range("slopes", d.slopes, d.q_heads * 4, 4);
    if (d.spans) c.range("spans", d.spans, n * 8, 8);
    if (d.tree) c.range("tree", d.tree, n * 8, 8);
    const uint64_t need = workspace_bytes(kv, d.batch.n_seqs, d.batch.n_tokens, d.q_heads);
    c.require(d.workspace_bytes >= need, "the workspace is smaller than t2i_kv_workspace_bytes");
    c.range("workspace", d.workspace, need, 256);
    if (!c.ok()) return T2I_ERR_INVALID;
    c.require(!overlap(d.out, c.token_bytes(n, d.q_heads, d.out_stride, 2), d.q, c.token_bytes(n, d.q_heads, d.q_stride, 2)),
              "out overlaps q");
    if (!c.ok()) return T2I_ERR_INVALID;
    a.pages = pages_of(kv, d.batch.table, d.batch.table_stride, d.batch.table_pages, d.batch.layer);
    a.q = d.q, a.out = d.out, a.lse = d.lse;
    a.q_stride = d.q_stride, a.out_stride = d.out_stride;
    a.slopes = d.slopes, a.spans = d.spans, a.tree = d.tree;
    a.q_heads = d.q_heads;
    a.group = d.q_heads / K;
    a.window = d.window;
    // (what a row of the table holds, where the caller does not say)
    a.max_len = d.max_len ? std::min(d.max_len, d.batch.table_pages << kv->token_shift) : d.batch.table_pages << kv->token_shift;
    a.scale = d.scale;
    a.softcap = d.softcap;
    const uint32_t no_loads = kv->timeout_countdown && --kv->timeout_countdown == 0;
    const KvLaunch l{&kv->map, d.workspace, kv->fault_dev, kv->sms, no_loads};
    const bool bf16 = kv->layout.dtype == T2I_BF16;
    return launch(kv, "kv_attend", [&] {
        if (uint64_t(a.group) * a.tok.max_new <= kFewRows) return bf16 ? launch_kv_few_bf16(a, l, stream) : launch_kv_few_f16(a, l, stream);
        return bf16 ? launch_kv_rows_bf16(a, l, stream) : launch_kv_rows_f16(a, l, stream);
    });
}

t2i_status commit(t2i_kv* kv, const t2i_kv_commit_desc& d, cudaStream_t stream) {
    Checks c(kv, "kv_commit");
    c.require(d.reserved == 0, "reserved must be 0");
    c.require(d.n_seqs <= 0x7FFFFFFFu && d.max_path <= 0x7FFFFFFFu, "too many sequences or path entries");
    if (!c.ok()) return T2I_ERR_INVALID;
    if (d.n_seqs == 0 || d.max_path == 0) return T2I_OK;
    const t2i_status past = past_fault(kv, "kv_commit");
    if (past != T2I_OK) return past;
    c.table(d.table, d.table_stride, d.table_pages, d.n_seqs);
    c.range("ctx", d.ctx, uint64_t(d.n_seqs) * 4, 4);
    c.range("path", d.path, uint64_t(d.n_seqs) * d.max_path * 4, 4);
    c.range("counts", d.counts, uint64_t(d.n_seqs) * 4, 4);
    if (!c.ok()) return T2I_ERR_INVALID;
    KvCommit a{};
    a.pages = pages_of(kv, d.table, d.table_stride, d.table_pages, 0);
    a.ctx = d.ctx, a.path = d.path, a.counts = d.counts;
    a.n_seqs = d.n_seqs;
    a.max_path = d.max_path;
    return launch(kv, "kv_commit", [&] { return launch_kv_commit(a, stream); });
}

using PFN_encodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                     const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                     CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The pool's pages for TMA (KvLaunch::map): null, or why not.
const char* encode_map(t2i_kv* kv) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
        return "the driver has no tensor maps";
    const t2i_kv_layout& l = kv->layout;
    const cuuint64_t dims[3] = {l.head_dim, (cuuint64_t(l.layers) * 2 * l.kv_heads) << kv->token_shift, kv->info.total_pages};
    const cuuint64_t strides[2] = {l.head_dim * 2u, kv->info.page_bytes};
    const cuuint32_t box[3] = {64, kv->token_shift < 7 ? 1u << kv->token_shift : 128u, 1};
    const cuuint32_t step[3] = {1, 1, 1};
    const CUresult r = reinterpret_cast<PFN_encodeTiled>(p)(
        &kv->map, l.dtype == T2I_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
        reinterpret_cast<void*>(kv->info.pool), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? nullptr : "the driver refuses a tensor map of the pool";
}

}  // namespace
}  // namespace t2i

extern "C" {

t2i_status t2i_kv_page_tokens(uint64_t page_bytes, const t2i_kv_layout* layout, uint32_t* out) {
    if (!layout || !out) {
        t2i::set_thread_error("t2i_kv_page_tokens: null layout or out");
        return T2I_ERR_INVALID;
    }
    *out = 0;
    if (const char* why = t2i::layout_error(*layout)) {
        t2i::set_thread_error(std::string("t2i_kv_page_tokens: ") + why);
        return T2I_ERR_INVALID;
    }
    const int s = t2i::page_token_shift(page_bytes, *layout);
    if (s < 0) {
        t2i::set_thread_error("t2i_kv_page_tokens: a page must hold the rows of at least 8 tokens (take larger pages, "
                              "or fewer layers to a page)");
        return T2I_ERR_INVALID;
    }
    *out = 1u << s;
    return T2I_OK;
}

t2i_status t2i_kv_create(t2i_store* store, const t2i_kv_layout* layout, t2i_kv** out) {
    if (!out) {
        t2i::set_thread_error("t2i_kv_create: null out");
        return T2I_ERR_INVALID;
    }
    *out = nullptr;
    if (!store || !layout) {
        t2i::set_thread_error("t2i_kv_create: null store or layout");
        return T2I_ERR_INVALID;
    }
    const t2i::StoreInfo info = t2i::store_info(store);
    uint32_t tokens = 0;
    const t2i_status st = t2i_kv_page_tokens(info.page_bytes, layout, &tokens);
    if (st != T2I_OK) return st;
    try {
        uint32_t shift = 0;
        while ((1u << shift) < tokens) ++shift;
        t2i::DeviceScope g(info.device);
        std::unique_ptr<t2i_kv> kv(new t2i_kv{});
        kv->store = store;
        kv->info = info;
        kv->layout = *layout;
        kv->token_shift = shift;
        int sms = 0;
        cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, info.device);
        kv->sms = uint32_t(sms);
        if (const char* why = e == cudaSuccess ? t2i::encode_map(kv.get()) : "cannot query the device") {
            t2i::set_thread_error(std::string("t2i_kv_create: ") + why);
            return T2I_ERR_CUDA;
        }
        e = cudaHostAlloc(reinterpret_cast<void**>(&kv->fault), sizeof(uint32_t), cudaHostAllocMapped);
        if (e == cudaSuccess) {
            *kv->fault = 0;
            e = cudaHostGetDevicePointer(reinterpret_cast<void**>(&kv->fault_dev), kv->fault, 0);
            if (e != cudaSuccess) cudaFreeHost(kv->fault);
        }
        if (e != cudaSuccess) {
            t2i::set_thread_error(std::string("t2i_kv_create: pinned host memory: ") + cudaGetErrorString(e));
            return T2I_ERR_CUDA;
        }
        *out = kv.release();
    } catch (const std::exception& e) {
        t2i::set_thread_error(std::string("t2i_kv_create: host error: ") + e.what());
        return T2I_ERR_INVALID;
    }
    return T2I_OK;
}

t2i_status t2i_kv_destroy(t2i_kv* kv) {
    if (!kv) return T2I_OK;
    t2i::DeviceScope g(kv->info.device);
    cudaFreeHost(kv->fault);  // (waits for kernels that may write it)
    delete kv;
    return T2I_OK;
}

#define T2I_KV_CALL(kv, desc, expr)                                          \
    do {                                                                     \
        if (!(kv)) return T2I_ERR_INVALID;                                   \
        t2i::Nvtx nvtx_range(__func__);                                      \
        std::lock_guard<std::mutex> lock(t2i::store_mutex((kv)->store));     \
        try {                                                                \
            if (!(desc)) {                                                   \
                t2i::store_set_error((kv)->store, "null descriptor");        \
                return T2I_ERR_INVALID;                                      \
            }                                                                \
            return (expr);                                                   \
        } catch (const std::exception& e) {                                  \
            t2i::store_set_error((kv)->store, std::string("host error: ") + e.what()); \
            return T2I_ERR_INVALID;                                          \
        }                                                                    \
    } while (0)

t2i_status t2i_kv_append(t2i_kv* kv, const t2i_kv_append_desc* desc, void* cuda_stream) {
    T2I_KV_CALL(kv, desc, t2i::append(kv, *desc, static_cast<cudaStream_t>(cuda_stream)));
}

t2i_status t2i_kv_attend(t2i_kv* kv, const t2i_kv_attend_desc* desc, void* cuda_stream) {
    T2I_KV_CALL(kv, desc, t2i::attend(kv, *desc, static_cast<cudaStream_t>(cuda_stream)));
}

t2i_status t2i_kv_commit(t2i_kv* kv, const t2i_kv_commit_desc* desc, void* cuda_stream) {
    T2I_KV_CALL(kv, desc, t2i::commit(kv, *desc, static_cast<cudaStream_t>(cuda_stream)));
}

t2i_status t2i_kv_workspace_bytes(const t2i_kv* kv, uint32_t n_seqs, uint32_t n_tokens, uint32_t q_heads, uint64_t* out) {
    if (!kv || !out) return T2I_ERR_INVALID;
    *out = t2i::workspace_bytes(kv, n_seqs, n_tokens, q_heads);
    return T2I_OK;
}

t2i_status t2i_kv_inject_timeout(t2i_kv* kv, uint32_t countdown) {
    if (!kv) return T2I_ERR_INVALID;
    std::lock_guard<std::mutex> lock(t2i::store_mutex(kv->store));
    kv->timeout_countdown = countdown;
    return T2I_OK;
}

}  // extern "C"
