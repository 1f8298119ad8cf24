// Entry points of rotary positions and of the paged cache of keys and values.
#include <cmath>

#include "ec_operators.h"

using namespace ec;

namespace {

constexpr int64_t kRotaryRowsMax = 1 << 24;
constexpr int kHeadsMax = 1024;           // heads of a row, in and out of the cache
constexpr int kRotaryHeadDimMax = 512;
constexpr int kKvRowsMax = 1 << 20;
constexpr int kSeqsMax = 65535;
constexpr int kKeysMax = 1 << 30;         // (the last chunk's end is an int)

// The strides of [rows, heads, head_dim] let no two elements of a tensor that is written meet.
bool apart(int64_t rows, int heads, int head_dim, size_t ld, size_t ld_head) {
  const size_t one = (size_t)head_dim;
  const bool heads_inside = (heads == 1 || ld_head >= one) && (rows == 1 || ld >= (heads == 1 ? 0 : (heads - 1) * ld_head) + one);
  const bool rows_inside = (rows == 1 || ld >= one) && (heads == 1 || ld_head >= (rows == 1 ? 0 : (size_t)(rows - 1) * ld) + one);
  return heads_inside || rows_inside;
}

const char* cache_error(const ec_kv_cache* c) {
  if (!c) return "cache must not be NULL";
  if (c->type != EC_T_BF16 && c->type != EC_T_E4M3) return "a cache is EC_T_BF16 or EC_T_E4M3";
  if (c->page != 32 && c->page != 64 && c->page != 128 && c->page != 256) return "page must be 32, 64, 128 or 256";
  if (c->pages < 1 || (int64_t)c->pages * c->page > INT32_MAX) return "pages must be 1 or more, with less than 2^31 tokens";
  if (c->kv_heads < 1 || c->kv_heads > kHeadsMax) return "kv_heads must be in [1, 1024]";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  return nullptr;
}
KvCache cache_of(const ec_kv_cache* c) {
  return {(uint8_t*)c->data, c->pages, c->page, c->kv_heads, c->head_dim, c->type == EC_T_E4M3};
}
int check_data(const ec_kv_cache* c) {
  return c->data && aligned(c->data, 256) ? EC_OK : op_fail(EC_ERR_ARG, "the cache's data is NULL or not 256-byte aligned");
}

KvAttention attention_of(const ec_kv_attention_cfg* a) {
  KvAttention k = {};
  k.rows = a->rows; k.heads = a->heads; k.seqs = a->seqs; k.max_rows = a->max_rows; k.max_keys = a->max_keys;
  k.table_ld = a->table_ld; k.prefix_len = a->prefix_len; k.causal = a->causal != 0; k.scale = a->scale;
  return k;
}
const char* attention_error(const ec_kv_cache* c, const ec_kv_attention_cfg* a) {
  if (!a) return "cfg must not be NULL";
  if (a->rows < 0 || a->rows > kKvRowsMax) return "rows must be in [0, 1048576]";
  if (a->heads < 1 || a->heads > kHeadsMax || a->heads % c->kv_heads) return "heads must be a multiple of kv_heads, at most 1024";
  if (a->seqs < 1 || a->seqs > kSeqsMax) return "seqs must be in [1, 65535]";
  if (a->max_rows < 0 || a->max_rows > a->rows) return "max_rows must be in [0, rows]";
  if (a->table_pages < 0 || (a->seqs > 1 && a->table_ld < (size_t)a->table_pages)) return "table_pages must not be negative, nor table_ld smaller";
  if (a->max_keys < 0 || a->max_keys > kKeysMax || a->max_keys > (int64_t)a->table_pages * c->page)
    return "max_keys must be in [0, table_pages * page], at most 2^30";
  if (a->prefix_pages < 0 || a->prefix_len < 0 || a->prefix_len > kKeysMax || a->prefix_len > (int64_t)a->prefix_pages * c->page)
    return "prefix_len must be in [0, prefix_pages * page], at most 2^30";
  if (!(a->scale > 0.f) || !(a->scale <= 1e38f)) return "scale must be positive, at most 1e38";
  const int64_t queries = (int64_t)a->max_rows * (a->heads / c->kv_heads);
  if ((queries + 15) / 16 * a->seqs * c->kv_heads > INT32_MAX / 1024) return "too many rows of too many sequences: give a smaller max_rows";
  return nullptr;
}

}  // namespace

extern "C" {

int ec_rotary_frequencies(const ec_rotary_cfg* cfg, double* turns) {
  if (!cfg || !turns) return op_fail(EC_ERR_ARG, "cfg and turns must not be NULL");
  if (cfg->dim < 2 || cfg->dim > kRotaryHeadDimMax || cfg->dim % 2) return op_fail(EC_ERR_ARG, "dim must be even, in [2, 512]");
  if (!(cfg->base > 0) || !std::isfinite(cfg->base)) return op_fail(EC_ERR_ARG, "base must be finite and positive");
  if (!(cfg->factor >= 1) || !std::isfinite(cfg->factor)) return op_fail(EC_ERR_ARG, "factor must be finite, 1 or more");
  if (!(cfg->original >= 0) || !std::isfinite(cfg->original)) return op_fail(EC_ERR_ARG, "original must be finite and not negative");
  if (cfg->original > 0 && !(cfg->high > cfg->low && std::isfinite(cfg->low) && std::isfinite(cfg->high)))
    return op_fail(EC_ERR_ARG, "low must be smaller than high");
  constexpr double kTurn = 6.283185307179586;
  for (int i = 0; i < cfg->dim / 2; ++i) {
    const double theta = std::pow(cfg->base, -2.0 * i / cfg->dim);
    double kept = 0;
    if (cfg->original > 0) kept = std::fmin(std::fmax((cfg->original * theta / kTurn - cfg->low) / (cfg->high - cfg->low), 0.0), 1.0);
    turns[i] = theta * (kept + (1 - kept) / cfg->factor) / kTurn;
  }
  return EC_OK;
}

int ec_rotary(const void* x, int32_t type, int64_t rows, int32_t heads, int32_t head_dim, size_t ld, size_t ld_head,
              const int32_t* positions, const double* turns, int32_t dim, int32_t interleaved, float amplitude, int32_t inverse, void* out,
              size_t out_ld, size_t out_ld_head, void* hip_stream) {
  if (!plain_type(type)) return op_fail(EC_ERR_ARG, "x must be EC_T_F32 or EC_T_BF16");
  if (rows < 0 || rows > kRotaryRowsMax) return op_fail(EC_ERR_ARG, "rows must be in [0, 16777216]");
  if (heads < 1 || heads > kHeadsMax) return op_fail(EC_ERR_ARG, "heads must be in [1, 1024]");
  if (head_dim < 2 || head_dim > kRotaryHeadDimMax) return op_fail(EC_ERR_ARG, "head_dim must be in [2, 512]");
  if (dim < 2 || dim > head_dim || dim % 2) return op_fail(EC_ERR_ARG, "dim must be even, in [2, head_dim]");
  if (!std::isfinite(amplitude)) return op_fail(EC_ERR_ARG, "amplitude must be finite");
  if (rows == 0) return EC_OK;
  if (!x || !positions || !turns || !out) return op_fail(EC_ERR_ARG, "x, positions, turns and out must not be NULL");
  if (!apart(rows, heads, head_dim, out_ld, out_ld_head)) return op_fail(EC_ERR_ARG, "out's rows and heads overlap");
  if (x == out && ((rows > 1 && ld != out_ld) || (heads > 1 && ld_head != out_ld_head)))
    return op_fail(EC_ERR_ARG, "in place, out's strides must be x's");
  if (!aligned(x, type_bytes(type)) || !aligned(out, type_bytes(type)) || !aligned(positions, 4) || !aligned(turns, 8))
    return op_fail(EC_ERR_ARG, "x, out, positions and turns must be aligned to their elements");
  launch_rotary(x, type == EC_T_BF16, rows, heads, head_dim, ld, ld_head, positions, turns, dim, interleaved != 0, amplitude, inverse != 0,
                out, out_ld, out_ld_head, (hipStream_t)hip_stream);
  return op_done("rotation kernel");
}

size_t ec_kv_bytes(const ec_kv_cache* cache) {
  return cache_error(cache) ? 0 : kv_bytes(cache_of(cache));
}

static int kv_move(const ec_kv_cache* cache, const void* k, const void* v, int32_t type, int32_t rows, const size_t (&ld)[4],
                   const int32_t* slots, bool out) {
  if (const char* what = cache_error(cache)) return op_fail(EC_ERR_ARG, what);
  if (!plain_type(type)) return op_fail(EC_ERR_ARG, "k and v must be EC_T_F32 or EC_T_BF16");
  if (rows < 0 || rows > kKvRowsMax) return op_fail(EC_ERR_ARG, "rows must be in [0, 1048576]");
  if (rows == 0) return EC_OK;
  const int rc = check_data(cache);
  if (rc != EC_OK) return rc;
  if (!k || !v || !slots) return op_fail(EC_ERR_ARG, "k, v and slots must not be NULL");
  if (!aligned(k, type_bytes(type)) || !aligned(v, type_bytes(type)) || !aligned(slots, 4))
    return op_fail(EC_ERR_ARG, "k, v and slots must be aligned to their elements");
  if (out && !(apart(rows, cache->kv_heads, cache->head_dim, ld[0], ld[1]) && apart(rows, cache->kv_heads, cache->head_dim, ld[2], ld[3])))
    return op_fail(EC_ERR_ARG, "rows and heads that are written overlap");
  return 1;
}

int ec_kv_write(const ec_kv_cache* cache, const void* k, const void* v, int32_t type, int32_t rows, size_t k_ld, size_t k_ld_head,
                size_t v_ld, size_t v_ld_head, const int32_t* slots, void* hip_stream) {
  const size_t ld[4] = {k_ld, k_ld_head, v_ld, v_ld_head};
  const int rc = kv_move(cache, k, v, type, rows, ld, slots, false);
  if (rc <= 0) return rc;
  launch_kv_write(cache_of(cache), k, v, type == EC_T_BF16, rows, ld, slots, (hipStream_t)hip_stream);
  return op_done("cache write kernel");
}

int ec_kv_read(const ec_kv_cache* cache, const int32_t* slots, int32_t rows, void* k, void* v, int32_t type, size_t k_ld,
               size_t k_ld_head, size_t v_ld, size_t v_ld_head, void* hip_stream) {
  const size_t ld[4] = {k_ld, k_ld_head, v_ld, v_ld_head};
  const int rc = kv_move(cache, k, v, type, rows, ld, slots, true);
  if (rc <= 0) return rc;
  launch_kv_read(cache_of(cache), k, v, type == EC_T_BF16, rows, ld, slots, (hipStream_t)hip_stream);
  return op_done("cache read kernel");
}

size_t ec_kv_attention_workspace_bytes(const ec_kv_cache* cache, const ec_kv_attention_cfg* cfg) {
  if (cache_error(cache) || attention_error(cache, cfg) || cfg->rows == 0 || cfg->max_rows == 0) return 0;
  return kv_attention_workspace(cache_of(cache), attention_of(cfg));
}

int ec_kv_attention(const ec_kv_cache* cache, const ec_kv_attention_cfg* cfg, const void* q, size_t q_ld, size_t q_ld_head,
                    const int32_t* table, const int32_t* lengths, const int32_t* starts, const int32_t* prefix, void* out, size_t out_ld,
                    size_t out_ld_head, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const char* what = cache_error(cache)) return op_fail(EC_ERR_ARG, what);
  if (const char* what = attention_error(cache, cfg)) return op_fail(EC_ERR_ARG, what);
  if (!starts && cfg->rows != (int64_t)cfg->max_rows * cfg->seqs)
    return op_fail(EC_ERR_ARG, "without starts, rows must be seqs * max_rows");
  if (cfg->rows == 0 || cfg->max_rows == 0) return EC_OK;
  const int rc = check_data(cache);
  if (rc != EC_OK) return rc;
  if (!q || !lengths || !out) return op_fail(EC_ERR_ARG, "q, lengths and out must not be NULL");
  if (!table && cfg->max_keys) return op_fail(EC_ERR_ARG, "table must not be NULL");
  if (!prefix && cfg->prefix_len) return op_fail(EC_ERR_ARG, "prefix must not be NULL");
  if (!aligned(table, 4) || !aligned(lengths, 4) || !aligned(starts, 4) || !aligned(prefix, 4))
    return op_fail(EC_ERR_ARG, "table, lengths, starts and prefix must be aligned to their elements");
  if (!aligned(q, 16) || !aligned(out, 16) || (q_ld | q_ld_head | out_ld | out_ld_head) % 8)
    return op_fail(EC_ERR_ARG, "q and out must be 16-byte aligned, with strides of multiples of 8 elements");
  if (!apart(cfg->rows, cfg->heads, cache->head_dim, out_ld, out_ld_head)) return op_fail(EC_ERR_ARG, "out's rows and heads overlap");
  if (const size_t need = ec_kv_attention_workspace_bytes(cache, cfg)) {
    if (!workspace || !aligned(workspace, 256)) return op_fail(EC_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need) return op_fail(EC_ERR_WORKSPACE, "workspace smaller than ec_kv_attention_workspace_bytes()");
  }
  KvAttention a = attention_of(cfg);
  a.q = (const bf16_t*)q; a.q_ld = q_ld; a.q_head = q_ld_head;
  a.out = (bf16_t*)out; a.out_ld = out_ld; a.out_head = out_ld_head;
  a.table = table; a.lengths = lengths; a.starts = starts; a.prefix = prefix;
  launch_kv_attention(cache_of(cache), a, workspace, (hipStream_t)hip_stream);
  return op_done("attention kernels");
}

}  // extern "C"
