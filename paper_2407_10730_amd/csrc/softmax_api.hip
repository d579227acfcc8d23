// softmax_api.hip -- C ABI of softmax attention, rotary positions and cache pages: validation, plans, launches.
#include <algorithm>
#include <cmath>
#include <new>

#include "seqmix_workspace.h"

using namespace cv;

struct seqmix_softmax_desc {
    seqmix_softmax_params p;
    seqmix_softmax_plan_info plan;
    int quantum = 0;  // of shares: log2 of keys
    Workspace ws;     // of plan.workspace_bytes
    bool counts = false;  // the step kernel's counts of parts that are done are zero, as every call leaves them
};
struct seqmix_rotary_desc {
    seqmix_rotary_params p;
};
struct seqmix_pages_desc {
    seqmix_pages_params p;
};

namespace {

// Heads of one call; more make 32-bit indices of a token's elements overflow.
constexpr int32_t kMaxHeads = 1 << 20;
// Rows and keys of a sequence: the kernels number a tile's rows and look for the next tiles' keys, up to 640 behind the last, in 32
// bits.
constexpr int64_t kMaxKeys = kMaxRows - 1023;
constexpr int kPackedShift = 10;
constexpr float kLog2E = 1.4426950408889634f;  // exponentials are powers of two

int log2_of(int32_t page) { return 31 - __builtin_clz((unsigned)page); }

// A cache of `pages` pages of `page` tokens has less than 2^31 rows.
int check_pages(int64_t pages, int32_t page) {
    if (pages < 1 || page < 1 || (page & (page - 1))) return CONV2D_E_INVALID;
    if (page > SEQMIX_MAX_PAGE || pages > kMaxRows / page) return CONV2D_E_UNSUPPORTED;
    return CONV2D_OK;
}
int check_table(int64_t max_pages, int32_t page) {
    if (max_pages < 1) return CONV2D_E_INVALID;
    return max_pages > kMaxRows / page ? CONV2D_E_UNSUPPORTED : CONV2D_OK;
}

// Rows, heads and pages (one: packed) of a cache of k or v do not overlap.
bool cache_ok(int64_t rows, int64_t heads, int64_t pages, int64_t row, int64_t head, int64_t page, int64_t dim) {
    if (!strides_ok(rows, row, heads, head, dim)) return false;
    return pages <= 1 || page >= (rows - 1) * row + (heads - 1) * head + dim;
}

// Heads that share a workgroup where sequences are short: as many of those that share a k/v head as fill its rows.
int32_t packed_heads(int64_t rows, int64_t length, int32_t rep) {
    int32_t pack = 1;
    for (int32_t d = 2; d <= rep; ++d)
        if (rep % d == 0 && d * length <= rows) pack = d;
    return pack;
}

// Where the tiles of rows are fewer than this, their keys are divided in shares, one for each workgroup that the card holds.
// 128 rows per tile, keys in a cache: 4 prompts of 300 to 700 tokens that go on from up to 12000, 16 heads of 128 (304 tiles):
// 194 us, by tiles 400; about as many keys as tokens, where tiles see half of them on average and the card overlaps short
// and long ones: 3 of 1000 tokens (384): 54 us, by tiles 42; one of 2200 (288): 61 and 62; 10 packed ones, 12 heads of 64 x 128
// (648): 71, by tiles 64; rows that are no multiple of 16 bytes alike (2048 tokens, 16 heads of 127, 272 tiles: 118, by tiles
// 110; of 63 53 and 56; 3 of 1000 tokens, heads of 127: 110 and 78); fp32 is slower by tiles (3 of 1300, 12 heads of 80 x 112:
// 222 us, by tiles 387).
// 32 rows: 64 single tokens over up to 8000 keys, 4 k/v heads (288): 111 us, by tiles 131; 2 over 65536 (8): 61 us, 700.
int64_t full_card(const seqmix_softmax_params& p, bool step) {
    if (step) return 4 * kSeqmixCUs;
    return p.dtype == CONV2D_BF16 && !p.page && p.key_tokens <= 2 * p.tokens ? kSeqmixCUs : 2 * kSeqmixCUs;
}
// ... and sequences are at most this many, as each wave looks at all of them.
constexpr int64_t kShareSeqs = 1024;
// Shares of the prompt kernel: as many workgroups as its registers allow, two per CU or, of dims padded to more than 256 together,
// one (the prompts above with heads of 256 428 us, with two 450; fp32, 3 of 1300 tokens, 12 heads of 80 x 112 222 with two, 269
// with one).  Of the step kernel, whose tiles fill LDS, one (2 tokens as above 68 us, with two 80).
int64_t shares_of(const seqmix_softmax_params& p, bool step) {
    auto padded = [](int32_t d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; };
    return step || padded(p.dk) + padded(p.dv) > 256 ? kSeqmixCUs : 2 * kSeqmixCUs;
}
// Quanta (64 keys, 128 in the step kernel) of a share at least, and of units that are not divided: beginning and joining parts
// costs some.  bf16 prompts (16 heads of 128): 600 tokens (10 quanta) whole 22 us, divided 27, 1000 (16) 33 and 31, 100 after 800
// (15) 32 and 26; shares of 3 at least: 1000 tokens 37, 100 after 800 21.  Single tokens: 4 over up to 1500 keys whole 17 us, in
// shares of 1 at least 12; 2 over 5000 in shares of 1, 2, 3 at least 16, 14, 18.  fp32, whose quanta take longer than all
// that: 300 tokens, 6 heads of 80 x 112, shares of 4 at least 66 us, of 2 40, of 1 28.
struct Division {
    int32_t least, whole;
};
Division division_of(bool step, int dtype) {
    if (dtype == CONV2D_F32) return {1, 1};
    return step ? Division{1, 6} : Division{4, 10};
}

int64_t part_bytes(const seqmix_softmax_params& p, bool step, int64_t rows) {
    return step ? rows * ((p.dv + 3) / 4 * 16 + 16) : (rows + 31) / 32 * ((p.dv + 7) / 8 * 1024 + 256);
}

void plan_softmax(seqmix_softmax_desc* d) {
    const seqmix_softmax_params& p = d->p;
    const int64_t length = std::max<int64_t>((p.tokens + p.seqs - 1) / p.seqs, 1);
    const int32_t rep = p.heads / p.kv_heads;
    const bool step = packed_heads(kStepRows, length, rep) == rep && length * rep <= kStepRows;
    const int32_t rows = step ? kStepRows : kPromptRows, pack = packed_heads(rows, length, rep);
    d->plan = seqmix_softmax_plan_info{step ? SEQMIX_KERNEL_STEP : SEQMIX_KERNEL_PROMPT, pack, 0, 0};
    const int64_t blocks = p.heads / pack, tiles = p.tokens / (rows / pack) + p.seqs;
    const int64_t keys = p.page ? p.max_pages * p.page : p.key_tokens;
    d->quantum = step ? 7 : 6;
    if (tiles * blocks < full_card(p, step) && p.seqs <= kShareSeqs && keys > (int64_t)division_of(step, p.dtype).whole << d->quantum) {
        d->plan.shares = shares_of(p, step);
        // quanta of all rows are counted in 32 bits
        for (; tiles * blocks * ((keys >> d->quantum) + 2) >= 1LL << 31;) ++d->quantum;
        d->plan.workspace_bytes = d->plan.shares * (2 * part_bytes(p, step, rows / pack * pack) + kMarkBytes);
    }
}

// What the kernels keep of each share behind the parts.
void* marks_of(const seqmix_softmax_desc* d) {
    return static_cast<char*>(d->ws.data) + d->plan.workspace_bytes - d->plan.shares * kMarkBytes;
}
bool counted(const seqmix_softmax_desc* d) { return d->plan.shares && d->plan.kernel == SEQMIX_KERNEL_STEP; }

__global__ __launch_bounds__(256) void clear_counts_kernel(uint32_t* counts, int n) {
    for (int i = threadIdx.x; i < n; i += 256) counts[i] = 0;
}

}  // namespace

extern "C" {

// ------------------------------------------------------------------ softmax attention
int seqmix_softmax_desc_create(const seqmix_softmax_params* params, seqmix_softmax_desc** out) {
    if (!params || !out) return CONV2D_E_NULL;
    const seqmix_softmax_params& p = *params;
    SM_TRY(check_seqs(p.tokens, p.seqs, p.slots));
    if (p.heads < 1 || p.kv_heads < 1 || p.heads % p.kv_heads != 0 || p.dk < 1 || p.dv < 1 || !std::isfinite(p.scale * kLog2E))
        return CONV2D_E_INVALID;
    if (p.mask < SEQMIX_MASK_FULL || p.mask > SEQMIX_MASK_TREE || !known_dtype(p.dtype) || p.dk > SEQMIX_MAX_HEAD_DIM ||
        p.dv > SEQMIX_MAX_HEAD_DIM || p.heads > kMaxHeads)
        return CONV2D_E_UNSUPPORTED;
    if (p.page) {
        SM_TRY(check_pages(p.pages, p.page));
        SM_TRY(check_table(p.max_pages, p.page));
    } else if (p.key_tokens < 0) {
        return CONV2D_E_INVALID;
    }
    if ((p.page ? p.max_pages * p.page : p.key_tokens) > kMaxKeys) return CONV2D_E_UNSUPPORTED;
    const int64_t rows = p.page ? p.page : p.key_tokens, pages = p.page ? p.pages : 1;
    if (!strides_ok(p.tokens, p.q_row, p.heads, p.q_head, p.dk) || !strides_ok(p.tokens, p.o_row, p.heads, p.o_head, p.dv) ||
        !cache_ok(rows, p.kv_heads, pages, p.k_row, p.k_head, p.k_page, p.dk) ||
        !cache_ok(rows, p.kv_heads, pages, p.v_row, p.v_head, p.v_page, p.dv))
        return CONV2D_E_INVALID;
    if ((p.tokens + p.seqs) * p.heads > kMaxKeys) return CONV2D_E_UNSUPPORTED;  // (workgroups too)
    seqmix_softmax_desc* d = new (std::nothrow) seqmix_softmax_desc;
    if (!d) return CONV2D_E_ALLOC;
    d->p = p;
    plan_softmax(d);
    *out = d;
    return CONV2D_OK;
}

int seqmix_softmax_desc_destroy(seqmix_softmax_desc* d) {
    if (!d) return CONV2D_OK;
    d->ws.release();
    delete d;
    return CONV2D_OK;
}

int seqmix_softmax_plan_query(const seqmix_softmax_desc* d, seqmix_softmax_plan_info* out) {
    if (!d || !out) return CONV2D_E_NULL;
    *out = d->plan;
    return CONV2D_OK;
}

int seqmix_softmax_reserve(seqmix_softmax_desc* d) {
    if (!d) return CONV2D_E_NULL;
    SM_TRY(d->ws.ensure(d->plan.workspace_bytes));
    if (!counted(d) || d->counts) return CONV2D_OK;
    if (hipMemset(marks_of(d), 0, (size_t)(d->plan.shares * kMarkBytes)) != hipSuccess || hipDeviceSynchronize() != hipSuccess)
        return CONV2D_E_HIP;
    d->counts = true;
    return CONV2D_OK;
}

int seqmix_softmax_fwd(seqmix_softmax_desc* d, const void* q, const void* k, const void* v, const int64_t* offsets,
                       const int64_t* key_offsets, const int32_t* slot_index, const int32_t* lens, const int32_t* table,
                       const int64_t* tree, void* o, void* stream) {
    if (!d) return CONV2D_E_NULL;
    const seqmix_softmax_params& p = d->p;
    if (p.tokens > 0 && (!q || !o || (p.mask == SEQMIX_MASK_TREE && !tree))) return CONV2D_E_NULL;
    if (p.tokens > 0 && (p.page ? !k || !v || !lens || !table : p.key_tokens > 0 && (!k || !v))) return CONV2D_E_NULL;
    SoftArgs a{};
    SM_TRY(seq_args(p.tokens, p.seqs, p.slots, offsets, slot_index, &a.sq));
    if (!p.page && !key_offsets && p.key_tokens != p.tokens) return CONV2D_E_INVALID;
    if (p.tokens == 0) return CONV2D_OK;
    a.q = q, a.k = k, a.v = v, a.o = o;
    a.koff = p.page ? nullptr : key_offsets;
    a.lens = lens, a.table = p.page ? table : nullptr, a.tree = tree;
    a.key_tokens = p.key_tokens, a.pages = p.page ? p.pages : 1, a.max_pages = p.max_pages;
    a.kp = {p.k_page, p.k_row, p.k_head};
    a.vp = {p.v_page, p.v_row, p.v_head};
    a.q_row = p.q_row, a.q_head = p.q_head, a.o_row = p.o_row, a.o_head = p.o_head;
    a.shift = p.page ? log2_of(p.page) : kPackedShift;
    if (!p.page) a.kp.page = p.k_row << kPackedShift, a.vp.page = p.v_row << kPackedShift;
    a.pack = d->plan.pack;
    a.blocks = p.heads / a.pack;
    a.by_rep = make_fastdiv((uint32_t)(p.heads / p.kv_heads));
    a.by_pack = make_fastdiv((uint32_t)a.pack);
    a.by_blocks = make_fastdiv((uint32_t)a.blocks);
    a.by_groups = make_fastdiv((uint32_t)((p.dv + 3) / 4));
    a.dk = p.dk, a.dv = p.dv, a.mask = p.mask;
    a.scale2 = std::fabs(p.scale) * kLog2E;
    a.qsign = !(a.scale2 > 0.0f) ? 0 : p.scale < 0.0f ? -1 : 1;
    if (a.qsign == 0) a.scale2 = 1.0f;
    const bool step = d->plan.kernel == SEQMIX_KERNEL_STEP;
    const int64_t unit = 16 / esize(p.dtype);
    // rows of k and v in 16-byte units
    const bool units = p.dk % unit == 0 && p.dv % unit == 0 && !(((uintptr_t)k | (uintptr_t)v) & 15) &&
                       !((p.k_row | p.k_head | p.k_page | p.v_row | p.v_head | p.v_page) % unit);
    a.near = p.dk >= unit && p.dv >= unit && (!p.page || p.page >= 8) && std::max(a.kp.page, a.vp.page) < (1LL << 28) &&
             std::max(p.k_row, p.v_row) < (1LL << 22);
    const bool vec = units && a.near;
    hipStream_t s = static_cast<hipStream_t>(stream);
    a.tile = (step ? kStepRows : kPromptRows) / a.pack;
    a.ids = seq_part_ids(a.sq, a.tile);
    if (d->plan.shares) {
        SM_TRY(d->ws.ensure(d->plan.workspace_bytes));
        SM_TRY(d->ws.order_after_last(s));
        if (counted(d) && !d->counts) {
            // (a captured call clears them whenever its graph runs, and for no other)
            hipLaunchKernelGGL(clear_counts_kernel, dim3(1), dim3(256), 0, s, static_cast<uint32_t*>(marks_of(d)), (int)d->plan.shares);
            if (hipGetLastError() != hipSuccess) return CONV2D_E_HIP;
            d->counts = Workspace::capture_of(s) == 0;
        }
        a.shares = (int32_t)d->plan.shares;
        a.quantum = d->quantum;
        a.grow = p.mask == SEQMIX_MASK_CAUSAL && a.tile % (1 << a.quantum) == 0 ? a.tile >> a.quantum : 0;
        a.least = division_of(step, p.dtype).least;
        a.whole = division_of(step, p.dtype).whole;
        a.most = (int32_t)((1LL << 31) / a.blocks - 1);
        a.ws = d->ws.data;
        a.marks = marks_of(d);
    }
    auto launch = p.dtype == CONV2D_BF16 ? (step ? launch_softmax_step_bf16 : launch_softmax_prompt_bf16)
                                         : (step ? launch_softmax_step_f32 : launch_softmax_prompt_f32);
    return launch(a, vec, s) == hipSuccess ? CONV2D_OK : CONV2D_E_HIP;
}

// ------------------------------------------------------------------ rotary positions
int seqmix_rotary_desc_create(const seqmix_rotary_params* params, seqmix_rotary_desc** out) {
    if (!params || !out) return CONV2D_E_NULL;
    const seqmix_rotary_params& p = *params;
    if (p.tokens < 0 || p.heads < 0 || p.kv_heads < 0 || p.dk < 1 || p.rot < 0 || p.rot % 2 != 0 || p.rot > p.dk)
        return CONV2D_E_INVALID;
    if (p.tokens > kMaxRows || p.heads > kMaxHeads || p.kv_heads > kMaxHeads || !known_dtype(p.dtype) ||
        p.dk > SEQMIX_MAX_HEAD_DIM || (p.layout != SEQMIX_ROTARY_HALF && p.layout != SEQMIX_ROTARY_INTERLEAVED))
        return CONV2D_E_UNSUPPORTED;
    if ((p.heads && (!strides_ok(p.tokens, p.q_row, p.heads, p.q_head, p.dk) ||
                     !strides_ok(p.tokens, p.qo_row, p.heads, p.qo_head, p.dk))) ||
        (p.kv_heads && (!strides_ok(p.tokens, p.k_row, p.kv_heads, p.k_head, p.dk) ||
                        !strides_ok(p.tokens, p.ko_row, p.kv_heads, p.ko_head, p.dk))))
        return CONV2D_E_INVALID;
    if (p.page) {
        if (p.kv_heads < 1 || p.dv < 1) return CONV2D_E_INVALID;
        if (p.dv > SEQMIX_MAX_HEAD_DIM) return CONV2D_E_UNSUPPORTED;
        SM_TRY(check_pages(p.pages, p.page));
        if (!strides_ok(p.tokens, p.v_row, p.kv_heads, p.v_head, p.dv) ||
            !cache_ok(p.page, p.kv_heads, p.pages, p.kc_row, p.kc_head, p.kc_page, p.dk) ||
            !cache_ok(p.page, p.kv_heads, p.pages, p.vc_row, p.vc_head, p.vc_page, p.dv))
            return CONV2D_E_INVALID;
    }
    seqmix_rotary_desc* d = new (std::nothrow) seqmix_rotary_desc{p};
    if (!d) return CONV2D_E_ALLOC;
    *out = d;
    return CONV2D_OK;
}

int seqmix_rotary_desc_destroy(seqmix_rotary_desc* d) {
    delete d;
    return CONV2D_OK;
}

int seqmix_rotary_fwd(const seqmix_rotary_desc* d, const void* q, const void* k, const void* v, const int32_t* position,
                      const double* freqs, void* q_out, void* k_out, void* k_cache, void* v_cache, const int32_t* place,
                      void* stream) {
    if (!d) return CONV2D_E_NULL;
    const seqmix_rotary_params& p = d->p;
    const bool cached = p.page > 0 && (k_cache || v_cache);
    const bool of_k = p.kv_heads > 0 && (k_out || (cached && k_cache));
    if (p.tokens > 0 && (!position || (p.rot && !freqs) || (p.heads && (!q || !q_out)) || (of_k && !k) ||
                         (cached && (!place || !k_cache || !v_cache || !v))))
        return CONV2D_E_NULL;
    if (p.tokens == 0) return CONV2D_OK;
    RotaryArgs a{};
    a.q = p.heads ? q : nullptr;
    a.k = of_k ? k : nullptr;
    a.v = v;
    a.qo = q_out;
    a.ko = p.kv_heads ? k_out : nullptr;
    a.kc = cached ? k_cache : nullptr;
    a.vc = cached ? v_cache : nullptr;
    a.position = position;
    a.place = cached ? place : nullptr;
    a.freqs = freqs;
    a.tokens = p.tokens;
    a.rows = p.page ? p.pages * p.page : 0;
    a.q_row = p.q_row, a.q_head = p.q_head, a.k_row = p.k_row, a.k_head = p.k_head, a.v_row = p.v_row, a.v_head = p.v_head;
    a.qo_row = p.qo_row, a.qo_head = p.qo_head, a.ko_row = p.ko_row, a.ko_head = p.ko_head;
    a.kp = {p.kc_page, p.kc_row, p.kc_head};
    a.vp = {p.vc_page, p.vc_row, p.vc_head};
    a.shift = p.page ? log2_of(p.page) : 0;
    a.heads = p.heads, a.kv_heads = p.kv_heads, a.dk = p.dk, a.dv = p.dv, a.rot = p.rot;
    a.amplitude = p.amplitude;
    a.past = p.tokens * (p.heads + (of_k ? p.kv_heads : 0)) * p.dk * esize(p.dtype) >= kPastBytes;
    return launch_rotary(a, p.dtype, p.layout, static_cast<hipStream_t>(stream)) == hipSuccess ? CONV2D_OK : CONV2D_E_HIP;
}

// ------------------------------------------------------------------ pages of the cache
int seqmix_pages_desc_create(const seqmix_pages_params* params, seqmix_pages_desc** out) {
    if (!params || !out) return CONV2D_E_NULL;
    const seqmix_pages_params& p = *params;
    SM_TRY(check_seqs(p.tokens, p.seqs, p.slots));
    SM_TRY(check_pages(p.pages, p.page));
    SM_TRY(check_table(p.max_pages, p.page));
    seqmix_pages_desc* d = new (std::nothrow) seqmix_pages_desc{p};
    if (!d) return CONV2D_E_ALLOC;
    *out = d;
    return CONV2D_OK;
}

int seqmix_pages_desc_destroy(seqmix_pages_desc* d) {
    delete d;
    return CONV2D_OK;
}

int seqmix_pages_fwd(const seqmix_pages_desc* d, const int32_t* kept, const int64_t* offsets, const int32_t* slot_index,
                     int32_t* lens, int32_t* table, int32_t* free_pages, int32_t* taken, int32_t* place, int32_t* position,
                     int32_t* admitted, void* stream) {
    if (!d) return CONV2D_E_NULL;
    const seqmix_pages_params& p = d->p;
    if (!lens || !table || !free_pages || !taken || !admitted || (p.tokens > 0 && (!place || !position))) return CONV2D_E_NULL;
    PagesArgs a{};
    SM_TRY(seq_args(p.tokens, p.seqs, p.slots, offsets, slot_index, &a.sq));
    a.kept = kept;
    a.lens = lens, a.table = table, a.free_pages = free_pages, a.taken = taken;
    a.place = place, a.position = position, a.admitted = admitted;
    a.pages = (int32_t)p.pages, a.max_pages = (int32_t)p.max_pages, a.shift = log2_of(p.page);
    a.by_len = make_fastdiv((uint32_t)std::max<int64_t>(a.sq.seq_len, 1));
    return launch_pages(a, static_cast<hipStream_t>(stream)) == hipSuccess ? CONV2D_OK : CONV2D_E_HIP;
}

}  // extern "C"
