// C entries of the 4-bit key/value cache: checks of the arguments, and how a call is cut into workgroups.
#include <limits.h>
#include <math.h>
#include <stdlib.h>

#include <algorithm>

#include "bnn_rotary.h"

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

bool weigh_takes(const Cache4& c, const Rows4& r, int group) {
    return (long long)r.tokens * group < (1LL << 30) && ((long long)r.table_pages << c.page_shift) <= (1LL << 30);
}

// How weights are added up.  Sequences of up to 32 rows by the kernel whose waves carry them, in as many workgroups as keep the chip busy with their loads (4096); of more by the one whose
// waves carry keys, with the rows of a tile of keys cut into parts until there are 2048 workgroups, 128 rows at least.  (Drafts of 30 rows: 20 us by the first, 34 by the second.  A chunk of 1024 rows over 1024 keys, 8 kv heads: parts
// of 128 rows 18 us, of 64 20, of 256 23.)
// Where sequences differ (start), the lengths of their runs being on the device, both are launched: the first has sequences of up to 64 rows, the second the others, of which there are at most as many as the call has rows
// for, in parts of 256 to 2048 rows, each of its workgroups looking for its own.  255 single tokens and a chunk of 4096 rows, 4000 keys: 235 us, all by the mean in one kernel 1790; 64 single tokens 30 instead of 28.  Where the second
// has so few workgroups that all run at once, it has the small sequences as well (2 to 36 tokens of 8 heads, 5 sequences: 17 us, both launches 29).
// Both go by the table's width: in one of 131072 tokens a chunk of 1024 tokens over 1024 keys has one part, 116 us in place of 35, and 255 single tokens and a prompt of 4000 take 3.2 ms in place of 0.31, nearly all workgroups finding nothing.
// near_rows: whether that kernel's offsets, of 2304 rows in 32 bits, reach (products of 24 bits); the other serves any distances, thousands of rows in runs.
WeighPlan4 plan_weigh(const Cache4& c, const Rows4& r, int dtype, int group, bool near_rows) {
    WeighPlan4 p = {};
    const long long all = (long long)r.tokens * group, rows = cdiv(all, r.batch), room = (long long)r.table_pages << c.page_shift, sequences = (long long)r.batch * c.kv_heads;
    const long long units = c.kv_heads * cdiv(room, 64 * cache4_weigh_tiles(c.dim));
    p.few_most = !near_rows ? INT_MAX : !r.start ? (rows <= 32 ? INT_MAX : -1) : rows > 32 && r.batch * units <= 768 ? -1 : 64;
    if (p.few_most >= 0) {
        p.runs = !near_rows && (r.start ? all : rows) > 256;
        p.row_tiles = rows > 16 && rows <= 32 && cache4_weigh_two(c.dim, dtype) && !p.runs ? 2 : 1;
        p.few_parts = (int)std::max(1LL, std::min(cdiv(4096, sequences), cdiv(room, 256)));
        p.few_groups = sequences * p.few_parts;
    }
    const long long many = p.few_most < 0 ? r.batch : std::min<long long>(r.batch, all / (p.few_most + 1LL));
    if (many > 0) {
        long long items = many, slots = 0;
        const bool one = r.batch * cdiv(room, 256) >= C4_THREADS / 256;      // (the joining launch does not reach)
        p.many_parts = 1;
        p.part_shift = 30;
        if (!r.start && !one) {
            p.many_parts = (int)std::max(1LL, std::min(cdiv(2048, units * many), cdiv(rows, 128)));
            slots = items = many * p.many_parts;
        } else if (r.start && !one) {
            p.part_shift = p.few_most < 0 ? 7 : 8;
            while (p.part_shift < 11 && (all * units) >> p.part_shift > 2048) ++p.part_shift;
            if (all > 1LL << p.part_shift) {
                items = many + (all >> p.part_shift);
                slots = 2 * (all >> p.part_shift);       // a sequence in several parts has more than 2^part_shift rows for every two of them
                p.many_parts = 2;            // at most, that is not 1
            }
        }
        if (items * c.kv_heads >= C4_THREADS) items = C4_THREADS;            // (refused by the groups)
        p.items = (int)std::min<long long>(items, INT_MAX);
        p.many_groups = items * units;
        p.slots = (int)std::min<long long>(slots, p.items);
        if (p.many_parts > 1) p.workspace_bytes = (size_t)p.slots * c.kv_heads * room * sizeof(float);
    }
    return p;
}

int make_rotation(const bnn_rotation* in, Rotation& rot) {
    if (!in || !in->frequencies || in->pairs < 1 || (in->neighbours != 0 && in->neighbours != 1) || (in->inverse != 0 && in->inverse != 1) || !isfinite(in->magnitude)) return BNN_ERR_INVALID_ARG;
    if (in->pairs > ROTARY_MAX_PAIRS) return BNN_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(in->frequencies) & 7u) || (reinterpret_cast<uintptr_t>(in->positions) & 3u)) return BNN_ERR_ALIGNMENT;
    rot.frequencies = in->frequencies;
    rot.positions = in->positions;
    rot.pairs = in->pairs;
    rot.magnitude = in->magnitude;
    rot.sign = in->inverse ? -1.0 : 1.0;
    return BNN_OK;
}

// Whether no two of n0 x n1 heads of dim elements, s0 and s1 elements apart, share an element.
bool heads_apart(long long n0, long long s0, long long n1, long long s1, int dim) {
    s0 = std::llabs(s0);
    s1 = std::llabs(s1);
    if ((n0 > 1 && s0 < dim) || (n1 > 1 && s1 < dim)) return false;
    if (n0 < 2 || n1 < 2) return true;
    if (s0 < s1) {
        std::swap(s0, s1);
        std::swap(n0, n1);
    }
    const __int128 reach = (__int128)(n1 - 1) * s1 + dim;            // of a row of the nearer ones
    for (long long i = 1; i < n0 && (__int128)i * s0 < reach; ++i) {         // (none, but for rows that reach into each other)
        const __int128 at = (__int128)i * s0, before = at / s1, past = at % s1;
        if ((before < n1 && past < dim) || (before + 1 < n1 && s1 - past < dim)) return false;
    }
    return true;
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

int bnn_rotary(const void* x, void* out, int dtype, int tokens, int heads, int dim, int64_t x_token, int64_t x_head, int64_t out_token, int64_t out_head,
               const bnn_rotation* rotation, void* stream) {
    Rotation rot;
    const int size = element_bytes(dtype);
    int rc = make_rotation(rotation, rot);
    if (rc != BNN_OK) return rc;
    if (size == 0 || tokens < 0 || heads < 0 || dim < 2 * rot.pairs) return BNN_ERR_INVALID_ARG;
    if (tokens == 0 || heads == 0) return BNN_OK;
    if (!x || !out || !rot.positions || (out == x && (out_token != x_token || out_head != x_head))) return BNN_ERR_INVALID_ARG;
    if (dim >= (1 << 20)) return BNN_ERR_UNSUPPORTED;
    if (!heads_apart(tokens, out_token, heads, out_head, dim)) return BNN_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(x) % size || reinterpret_cast<uintptr_t>(out) % size) return BNN_ERR_ALIGNMENT;
    const int width = rotary_width(size, {rot.pairs, dim - 2 * rot.pairs, x_token, x_head, out_token, out_head}, {x, out});
    return launch_rotary(x, out, dtype, tokens, heads, dim, x_token, x_head, out_token, out_head, width, rot, rotation->neighbours, static_cast<hipStream_t>(stream));
}

int bnn_cache4_write_rotary(const bnn_cache4* cache, const bnn_cache4_rows* rows, const bnn_rotation* rotation, const void* q, int64_t q_token, int64_t q_head, int heads, void* q_out,
                            const void* k, const void* v, int dtype, int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void* stream) {
    WriteRotary4 a = {};
    int rc = make_cache(cache, a.c);
    if (rc != BNN_OK || (rc = make_rows(rows, a.c, a.r)) != BNN_OK || (rc = make_rotation(rotation, a.rot)) != BNN_OK) return rc;
    if (element_bytes(dtype) == 0 || heads < 0 || 2 * a.rot.pairs > a.c.dim) return BNN_ERR_INVALID_ARG;
    if (a.r.tokens == 0) return BNN_OK;
    if ((rc = check_elements(k, dtype, k_token, k_head)) != BNN_OK || (rc = check_elements(v, dtype, v_token, v_head)) != BNN_OK) return rc;
    if (heads > 0 && ((rc = check_elements(q, dtype, q_token, q_head)) != BNN_OK || (rc = check_elements(q_out, dtype, 0, 0)) != BNN_OK)) return rc;
    if (heads > 0 && q_out == q && ((heads > 1 && q_head != a.c.dim) || (a.r.tokens > 1 && q_token != (int64_t)heads * a.c.dim))) return BNN_ERR_INVALID_ARG;
    if (heads > (1 << 30)) return BNN_ERR_UNSUPPORTED;
    a.q = q; a.q_token = q_token; a.q_head = q_head; a.q_out = q_out; a.heads = heads;
    a.k = k; a.k_token = k_token; a.k_head = k_head;
    a.v = v; a.v_token = v_token; a.v_head = v_head;
    int width = 8;
    while (a.rot.pairs % width != 0) width /= 2;             // (pointers and distances are multiples of 16 bytes, head_dim of 32)
    return launch_cache4_write_rotary(a, dtype, rotation->neighbours, width, static_cast<hipStream_t>(stream));
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

size_t bnn_cache4_weigh_workspace_bytes(const bnn_cache4* cache, const bnn_cache4_rows* rows, int dtype, int heads) {
    Cache4 c;
    Rows4 r;
    int group;
    if (make_cache(cache, c) != BNN_OK || make_rows(rows, c, r) != BNN_OK || check_heads(c, heads, group) != BNN_OK || element_bytes(dtype) == 0) return 0;
    return r.tokens == 0 || !weigh_takes(c, r, group) ? 0 : plan_weigh(c, r, dtype, group, true).workspace_bytes;
}

int bnn_cache4_weigh(const bnn_cache4* cache, const bnn_cache4_rows* rows, const void* q, int dtype, int64_t q_token, int64_t q_head, int heads, const float* lse,
                     float scale, int causal, int window, const float* previous, float decay, float* weights, int64_t width, void* workspace, size_t workspace_bytes, void* stream) {
    Weigh4 a = {};
    int rc = make_cache(cache, a.c);
    if (rc != BNN_OK || (rc = make_rows(rows, a.c, a.r)) != BNN_OK || (rc = check_heads(a.c, heads, a.group)) != BNN_OK) return rc;
    a.scale2 = scale * 1.4426950408889634f;
    a.unscale = (1.5 - 0.5 * a.scale2 / (scale * 1.4426950408889634)) / scale;       // (1 - e / 2) / scale, scale2 being (1 + e) scale / log 2
    if (element_bytes(dtype) == 0 || !(scale > 0.f) || !isfinite(a.scale2) || !isfinite(1.f / scale) || window < 0 || (window > 0 && !causal) || !isfinite(decay)) return BNN_ERR_INVALID_ARG;
    if (a.r.tokens == 0) return BNN_OK;
    if (!weights || !lse || width < ((long long)a.r.table_pages << a.c.page_shift)) return BNN_ERR_INVALID_ARG;
    if ((rc = check_elements(q, dtype, q_token, q_head)) != BNN_OK) return rc;
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(previous) & 3u) || (reinterpret_cast<uintptr_t>(weights) & 3u)) return BNN_ERR_ALIGNMENT;
    if (!weigh_takes(a.c, a.r, a.group)) return BNN_ERR_UNSUPPORTED;
    const long long far = 1LL << 24;
    const bool near_rows = q_token >= 0 && q_head >= 0 && q_token < far && q_head < far && a.group < far &&
                           ((2304 / a.group + 2) * q_token + a.group * q_head + a.c.dim) * element_bytes(dtype) < (1LL << 32);
    const WeighPlan4 p = plan_weigh(a.c, a.r, dtype, a.group, near_rows);
    if (std::max(p.few_groups, p.many_groups) >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    if (p.workspace_bytes != 0 && (!workspace || workspace_bytes < p.workspace_bytes)) return BNN_ERR_WORKSPACE;
    if (p.workspace_bytes != 0 && !aligned16(workspace)) return BNN_ERR_ALIGNMENT;
    a.q = q; a.q_token = q_token; a.q_head = q_head;
    a.div_group = make_fastdiv((uint32_t)a.group);
    a.div_heads = make_fastdiv((uint32_t)a.c.kv_heads);
    a.causal = causal ? 1 : 0;
    a.window = window;
    a.lse = lse; a.previous = previous; a.decay = decay; a.out = weights; a.width = width;
    a.few_most = p.few_most;
    a.items = p.items;
    a.slots = p.slots;
    a.part_shift = p.part_shift;
    if (p.items > 0) a.div_items = make_fastdiv((uint32_t)p.items);
    a.partial = static_cast<float*>(workspace);
    a.width4 = (long long)a.r.table_pages << a.c.page_shift;
    return launch_cache4_weigh(a, p, dtype, static_cast<hipStream_t>(stream));
}

size_t bnn_cache4_heaviest_workspace_bytes(const bnn_cache4* cache, int batch, int table_pages) {
    Cache4 c;
    if (make_cache(cache, c) != BNN_OK || batch < 1 || table_pages < 1 || ((long long)table_pages << c.page_shift) > (1LL << 30)) return 0;
    return plan_cache4_heaviest(c, batch, table_pages).workspace_bytes;
}

int bnn_cache4_heaviest(const bnn_cache4* cache, const int32_t* table, const int32_t* lens, int batch, int table_pages, const float* weights, int64_t width,
                        int keep, int first, int last, int32_t* tokens, int32_t* kept, void* workspace, size_t workspace_bytes, void* stream) {
    Heaviest4 a = {};
    const int rc = make_cache(cache, a.c);
    if (rc != BNN_OK) return rc;
    if (batch < 0 || table_pages < 0 || keep < 1 || first < 0 || last < 0 || (long long)first + last > keep) return BNN_ERR_INVALID_ARG;
    if (batch == 0) return BNN_OK;
    if (table_pages < 1 || !table || !lens || !weights || !tokens || !kept || width < ((long long)table_pages << a.c.page_shift)) return BNN_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(table) & 3u) || (reinterpret_cast<uintptr_t>(lens) & 3u) || (reinterpret_cast<uintptr_t>(weights) & 3u) ||
        (reinterpret_cast<uintptr_t>(tokens) & 3u) || (reinterpret_cast<uintptr_t>(kept) & 3u))
        return BNN_ERR_ALIGNMENT;
    if (batch >= C4_THREADS / 1024 || ((long long)table_pages << a.c.page_shift) > (1LL << 30)) return BNN_ERR_UNSUPPORTED;
    a.weights = weights; a.width = width;
    a.table = table; a.lens = lens; a.batch = batch; a.table_pages = table_pages;
    a.keep = keep; a.first = first; a.last = last;
    a.tokens = tokens; a.kept = kept;
    const HeaviestPlan4 p = plan_cache4_heaviest(a.c, batch, table_pages);
    if (p.workspace_bytes != 0 && (!workspace || workspace_bytes < p.workspace_bytes)) return BNN_ERR_WORKSPACE;
    if (p.workspace_bytes != 0 && !aligned16(workspace)) return BNN_ERR_ALIGNMENT;
    return launch_cache4_heaviest(a, p, workspace, static_cast<hipStream_t>(stream));
}

int bnn_cache4_move(const bnn_cache4* cache, const int32_t* tokens, int keep, const int32_t* table, int table_pages, const int32_t* into, int into_pages, int batch,
                    const float* weights, int64_t width, float* moved, void* stream) {
    Move4 a = {};
    const int rc = make_cache(cache, a.c);
    if (rc != BNN_OK) return rc;
    if (batch < 0 || table_pages < 0 || into_pages < 0 || keep < 1 || (weights ? width < 1 || !moved : moved != nullptr)) return BNN_ERR_INVALID_ARG;
    if (batch == 0 || into_pages == 0) return BNN_OK;
    if (table_pages < 1 || !tokens || !table || !into) return BNN_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(table) & 3u) || (reinterpret_cast<uintptr_t>(into) & 3u) || (reinterpret_cast<uintptr_t>(weights) & 3u) ||
        (reinterpret_cast<uintptr_t>(tokens) & 3u) || (reinterpret_cast<uintptr_t>(moved) & 3u))
        return BNN_ERR_ALIGNMENT;
    if (((long long)table_pages << a.c.page_shift) > (1LL << 30) || ((long long)into_pages << a.c.page_shift) > (1LL << 30)) return BNN_ERR_UNSUPPORTED;
    a.tokens = tokens; a.keep = keep;
    a.table = table; a.into = into; a.batch = batch; a.table_pages = table_pages; a.into_pages = into_pages;
    a.weights = weights; a.width = width; a.moved = moved;
    return launch_cache4_move(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
