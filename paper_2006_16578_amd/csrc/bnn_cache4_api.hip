// C entries of the 4-bit key/value cache: checks of the arguments, and how a call is cut into workgroups.
#include <math.h>

#include <algorithm>

#include "bnn_cache4.h"

using namespace bnn;

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool known_dim(int d) { return d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }
bool known_page(int p) { return p >= 16 && p <= 256 && (p & (p - 1)) == 0; }
int element_bytes(int dtype) { return dtype == BNN_F32 ? 4 : dtype == BNN_BF16 || dtype == BNN_F16 ? 2 : 0; }

int make_cache(const bnn_cache4* in, Cache4& c) {
    if (!in || !in->data || in->pages < 1 || in->kv_heads < 1 || (in->signs != 0 && in->signs != 1)) return BNN_ERR_INVALID_ARG;
    if (in->pages >= (1LL << 31) || in->kv_heads > 65535 || !known_dim(in->head_dim) || !known_page(in->page)) return BNN_ERR_UNSUPPORTED;
    if (!aligned16(in->data)) return BNN_ERR_ALIGNMENT;
    c.data = static_cast<uint8_t*>(in->data);
    c.pages = (int)in->pages;
    c.kv_heads = in->kv_heads;
    c.dim = in->head_dim;
    c.page = in->page;
    c.page_shift = 0;
    while ((1 << c.page_shift) < in->page) ++c.page_shift;
    const int codes = in->page * in->head_dim / 2, exps = in->page * in->head_dim / C4_GROUP;
    c.v_codes = codes;
    c.k_exps = 2 * codes;
    c.v_exps = 2 * codes + exps;
    c.signs = in->signs ? 2 * codes + 2 * exps : 0;
    c.record = (int)bnn_cache4_record_bytes(in->head_dim, in->page, in->signs);
    return BNN_OK;
}

int make_rows(const bnn_cache4_rows* in, const Cache4& c, Rows4& r) {
    if (!in || in->batch < 0 || in->tokens < 0 || in->table_pages < 0) return BNN_ERR_INVALID_ARG;
    r = {};
    r.tokens = in->tokens;
    if (in->tokens == 0) return BNN_OK;
    if (in->batch < 1 || in->table_pages < 1 || !in->table || !in->lens) return BNN_ERR_INVALID_ARG;
    if (!in->start && in->tokens % in->batch != 0) return BNN_ERR_INVALID_ARG;
    if (((long long)in->table_pages << c.page_shift) >= (1LL << 31)) return BNN_ERR_UNSUPPORTED;
    r.table = in->table;
    r.lens = in->lens;
    r.start = in->start;
    r.batch = in->batch;
    r.table_pages = in->table_pages;
    r.each = in->start ? 0 : in->tokens / in->batch;
    r.div_each = make_fastdiv((uint32_t)std::max(r.each, 1));
    return BNN_OK;
}

// Elements [tokens][heads][dim] that kernels read 16 bytes at a time.
int check_elements(const void* p, int dtype, int64_t token, int64_t head) {
    const int size = element_bytes(dtype);
    if (!p || size == 0) return BNN_ERR_INVALID_ARG;
    if (!aligned16(p) || token * size % 16 != 0 || head * size % 16 != 0) return BNN_ERR_ALIGNMENT;
    return BNN_OK;
}

// How attention is cut up.  Rows of a workgroup: 64 or 128 where the rows of a sequence fill them, else 16, or 32 where that saves a workgroup; by the mean over the batch, one
// choice for the launch, so single tokens beside a long chunk go through the kernel for many rows.  Parts of the keys: as many as 512 workgroups make, but of 2048 keys at
// least, by the table's width (lengths are known on the device only): a table much wider than its sequences leaves them fewer parts.  512 workgroups of eight waves are two to
// a compute unit for heads of 64 and for bf16 ones of 128; others take more than 128 registers, or more than 80 KB of LDS, and run one after another.  64 conversations of up to 8192 tokens, 8 kv heads: one part 66 us, with two
// 82 (before K's exponents were loaded four keys at a time, now one part 60); two documents of up to 131072: 32 parts 48 us, 48 parts 56, 64 parts 50; 5 drafted tokens over 1000 keys in one part 15 us, in two 19; one conversation of 777 tokens in
// one part 8.2 us, in two 10.7.
AttendPlan4 plan_attend(const Cache4& c, const Rows4& r, int dtype, int group, int window, int keep) {
    AttendPlan4 p = {};
    long long tiles, steps;
    if (keep > 0) {
        p.rows = 16;
        p.threads = 64 * cache4_waves(c.dim, dtype, 1);
        tiles = (long long)r.tokens * cdiv(group, 16);
        steps = cdiv((long long)keep * (c.page / 16), 2);
    } else {
        const long long rows = cdiv((long long)r.tokens * group, r.batch);
        const int wide = 64 * cache4_wide_qtiles(c.dim, dtype);
        p.rows = rows >= 64 ? wide : rows > 16 ? 16 * cache4_qtiles(c.dim, dtype) : 16;
        p.threads = rows >= 64 ? 256 : 64 * cache4_waves(c.dim, dtype, p.rows / 16);
        tiles = c4_tiles(r, group, p.rows, &p.seq_tiles);
        long long keys = (long long)r.table_pages << c.page_shift;
        if (window > 0) keys = std::min(keys, (long long)window + cdiv(p.rows, group) + 64);
        steps = cdiv(keys, 32);
    }
    const long long units = tiles * c.kv_heads;
    const long long splits = std::max(1LL, std::min(512 / units, cdiv(steps, 64)));
    p.chunk = (int)(cdiv(cdiv(steps, splits), 8) * 8);
    p.splits = (int)cdiv(steps, p.chunk);
    p.tiles = (int)std::min(tiles, (long long)INT32_MAX);
    if (p.splits > 1) {
        const size_t rows = (size_t)tiles * c.kv_heads * p.splits * p.rows;
        p.part_bytes = rows * c.dim * 4;
        p.workspace_bytes = p.part_bytes + rows * sizeof(f32x4);
    }
    return p;
}

int check_heads(const Cache4& c, int heads, int& group) {
    if (heads < 1 || heads % c.kv_heads != 0) return BNN_ERR_INVALID_ARG;
    group = heads / c.kv_heads;
    return BNN_OK;
}

}  // namespace

extern "C" {

size_t bnn_cache4_record_bytes(int head_dim, int page, int signs) {
    if (!known_dim(head_dim) || !known_page(page)) return 0;
    return (size_t)page * (head_dim + 2 * head_dim / C4_GROUP + (signs ? head_dim / 8 : 0));
}

int bnn_cache4_write(const bnn_cache4* cache, const bnn_cache4_rows* rows, const void* k, const void* v, int dtype,
                     int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void* stream) {
    Cache4 c;
    Rows4 r;
    int rc = make_cache(cache, c);
    if (rc != BNN_OK || (rc = make_rows(rows, c, r)) != BNN_OK) return rc;
    if (element_bytes(dtype) == 0) return BNN_ERR_INVALID_ARG;
    if (r.tokens == 0) return BNN_OK;
    if ((rc = check_elements(k, dtype, k_token, k_head)) != BNN_OK || (rc = check_elements(v, dtype, v_token, v_head)) != BNN_OK) return rc;
    if (cache4_row_blocks(c, r) * 256 >= C4_THREADS) return BNN_ERR_UNSUPPORTED;
    return launch_cache4_write(c, r, k, v, dtype, k_token, k_head, v_token, v_head, static_cast<hipStream_t>(stream));
}

int bnn_cache4_read(const bnn_cache4* cache, const bnn_cache4_rows* rows, void* k, void* v, int dtype, void* stream) {
    Cache4 c;
    Rows4 r;
    int rc = make_cache(cache, c);
    if (rc != BNN_OK || (rc = make_rows(rows, c, r)) != BNN_OK) return rc;
    if (element_bytes(dtype) == 0) return BNN_ERR_INVALID_ARG;
    if (r.tokens == 0) return BNN_OK;
    if ((rc = check_elements(k, dtype, 0, 0)) != BNN_OK || (rc = check_elements(v, dtype, 0, 0)) != BNN_OK) return rc;
    if (cache4_row_blocks(c, r) * 256 >= C4_THREADS) return BNN_ERR_UNSUPPORTED;
    return launch_cache4_read(c, r, k, v, dtype, static_cast<hipStream_t>(stream));
}

size_t bnn_cache4_select_workspace_bytes(const bnn_cache4* cache, const bnn_cache4_rows* rows) {
    Cache4 c;
    Rows4 r;
    if (make_cache(cache, c) != BNN_OK || make_rows(rows, c, r) != BNN_OK) return 0;
    return (size_t)r.tokens * c.kv_heads * r.table_pages * sizeof(uint16_t);
}

int bnn_cache4_select(const bnn_cache4* cache, const bnn_cache4_rows* rows, const void* q, int dtype, int64_t q_token, int64_t q_head, int heads,
                      int keep, int first, int last, int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
    Select4 a = {};
    int rc = make_cache(cache, a.c);
    if (rc != BNN_OK || (rc = make_rows(rows, a.c, a.r)) != BNN_OK || (rc = check_heads(a.c, heads, a.group)) != BNN_OK) return rc;
    if (!a.c.signs || element_bytes(dtype) == 0 || keep < 1 || first < 0 || last < 0 || (long long)first + last > keep) return BNN_ERR_INVALID_ARG;
    if ((long long)a.group * a.c.dim > 16000) return BNN_ERR_UNSUPPORTED;
    if (a.r.tokens == 0) return BNN_OK;
    if (!blocks) return BNN_ERR_INVALID_ARG;
    if ((rc = check_elements(q, dtype, q_token, q_head)) != BNN_OK) return rc;
    if ((long long)a.r.tokens * a.c.kv_heads >= (1LL << 24)) return BNN_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < bnn_cache4_select_workspace_bytes(cache, rows)) return BNN_ERR_WORKSPACE;
    if (!aligned16(workspace) || (reinterpret_cast<uintptr_t>(blocks) & 3u)) return BNN_ERR_ALIGNMENT;
    a.q = q; a.q_token = q_token; a.q_head = q_head;
    a.keep = keep; a.first = first; a.last = last; a.blocks = blocks;
    a.scores = static_cast<uint16_t*>(workspace);
    return launch_cache4_select(a, dtype, static_cast<hipStream_t>(stream));
}

size_t bnn_cache4_attend_workspace_bytes(const bnn_cache4* cache, const bnn_cache4_rows* rows, int dtype, int heads, int window, int keep) {
    Cache4 c;
    Rows4 r;
    int group;
    if (make_cache(cache, c) != BNN_OK || make_rows(rows, c, r) != BNN_OK || check_heads(c, heads, group) != BNN_OK || element_bytes(dtype) == 0) return 0;
    return r.tokens == 0 ? 0 : plan_attend(c, r, dtype, group, window, keep).workspace_bytes;
}

int bnn_cache4_attend(const bnn_cache4* cache, const bnn_cache4_rows* rows, const void* q, int dtype, int64_t q_token, int64_t q_head, int heads,
                      float scale, int causal, int window, const int32_t* blocks, int keep, void* out, float* lse,
                      void* workspace, size_t workspace_bytes, void* stream) {
    Attend4 a = {};
    int rc = make_cache(cache, a.c);
    if (rc != BNN_OK || (rc = make_rows(rows, a.c, a.r)) != BNN_OK || (rc = check_heads(a.c, heads, a.group)) != BNN_OK) return rc;
    const float scale2 = scale * 1.4426950408889634f;                // for powers of two
    if (element_bytes(dtype) == 0 || !(scale > 0.f) || !isfinite(scale2) || window < 0 || (window > 0 && !causal)) return BNN_ERR_INVALID_ARG;
    if (blocks ? keep < 1 : keep < 0) return BNN_ERR_INVALID_ARG;
    if (a.r.tokens == 0) return BNN_OK;
    if (!blocks && keep != 0) return BNN_ERR_INVALID_ARG;            // (the lists of no rows need no memory)
    if ((rc = check_elements(q, dtype, q_token, q_head)) != BNN_OK || (rc = check_elements(out, dtype, 0, 0)) != BNN_OK) return rc;
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(blocks) & 3u)) return BNN_ERR_ALIGNMENT;
    if ((long long)a.r.tokens * a.group >= (1LL << 30) || (long long)keep * a.c.page >= (1LL << 31)) return BNN_ERR_UNSUPPORTED;
    const AttendPlan4 p = plan_attend(a.c, a.r, dtype, a.group, window, keep);
    if ((long long)p.tiles * p.splits * a.c.kv_heads >= C4_THREADS / p.threads) return BNN_ERR_UNSUPPORTED;
    if (p.workspace_bytes != 0 && (!workspace || workspace_bytes < p.workspace_bytes)) return BNN_ERR_WORKSPACE;
    if (p.workspace_bytes != 0 && !aligned16(workspace)) return BNN_ERR_ALIGNMENT;
    a.q = q; a.q_token = q_token; a.q_head = q_head;
    a.div_group = make_fastdiv((uint32_t)a.group);
    a.scale = scale2;
    a.causal = causal ? 1 : 0;
    a.window = window;
    a.blocks = blocks; a.keep = keep;
    a.out = out; a.lse = lse;
    a.tiles = p.tiles; a.seq_tiles = p.seq_tiles; a.div_seq_tiles = make_fastdiv((uint32_t)std::max(p.seq_tiles, 1));
    a.splits = p.splits; a.chunk = p.chunk;
    a.div_splits = make_fastdiv((uint32_t)p.splits);
    a.div_heads = make_fastdiv((uint32_t)a.c.kv_heads);
    a.part = static_cast<float*>(workspace);
    a.part_sums = reinterpret_cast<f32x4*>(static_cast<char*>(workspace) + p.part_bytes);
    hipStream_t s = static_cast<hipStream_t>(stream);
    switch (a.c.dim) {
        case 64: return launch_cache4_attend64(a, dtype, p.rows, s);
        case 96: return launch_cache4_attend96(a, dtype, p.rows, s);
        case 128: return launch_cache4_attend128(a, dtype, p.rows, s);
        case 192: return launch_cache4_attend192(a, dtype, p.rows, s);
        default: return launch_cache4_attend256(a, dtype, p.rows, s);
    }
}

}  // extern "C"
