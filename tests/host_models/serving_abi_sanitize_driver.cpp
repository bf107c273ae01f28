// The host code of the entry points around a serving loop's attention calls (norm and rotation, decode behind a shared prefix, decode
// with weights, eviction) under the sanitizers: only calls that are refused before anything is enqueued, and workspace sizes.
// Exit code 0 = every call returned the documented status and the sanitizers saw nothing.
#include <cstdint>
#include <cstdio>
#include <limits>

#include "../../include/slimattn.h"

static int bad = 0;
static void expect(int got, int want, const char* what) {
    if (got != want) {
        std::fprintf(stderr, "serving_abi_sanitize_driver: %s: status %d, expected %d\n", what, got, want);
        ++bad;
    }
}

// aligned addresses 2^40 apart, never dereferenced
static void* at(int i, int off = 0) { return reinterpret_cast<void*>((static_cast<uintptr_t>(i + 1) << 40) + off); }
static float* fl(int i, int off = 0) { return static_cast<float*>(at(i, off)); }
static int8_t* by(int i, int off = 0) { return static_cast<int8_t*>(at(i, off)); }
static int32_t* in(int i, int off = 0) { return static_cast<int32_t*>(at(i, off)); }

static int rotate(int64_t qs, int batch, int seq, int d, int table, int pairs, double eps, void* q_out) {
    return slim_qk_norm_rope(at(0), at(1), at(2), qs, 1024, 1024, nullptr, nullptr, fl(3), in(4), q_out, at(6), at(7), batch, 8, 8, seq, d, table,
                             pairs, eps, nullptr);
}
static int append(int kv_len, int32_t* slots, float* v_scale) {
    return slim_qk_norm_rope_append_int8(at(0), at(1), at(2), 1024, 1024, 1024, at(3), at(4), fl(5), in(6), slots, at(8), by(9), fl(10), by(11),
                                         v_scale, 2, 8, 8, 3, kv_len, 128, 100, 0, 1e-6, nullptr);
}
static int prefix(size_t bytes, int batch, int prefix_len, int kv_len, float scale, void* out) {
    return slim_attn_decode_int8_shared_prefix(at(0), by(1), fl(2), by(3), fl(4), by(5), fl(6), by(7), fl(8), in(9), out, at(11), bytes, batch, 64, 8,
                                               prefix_len, kv_len, 128, 1, scale, nullptr);
}
static int weights(size_t bytes, int batch, int kv_len, float* w_in, float* w_out) {
    return slim_attn_decode_int8_weights(at(0), by(1), fl(2), by(3), fl(4), in(5), w_in, w_out, at(8), at(9), bytes, batch, 64, 8, kv_len, 128, 1, 0.1f,
                                         nullptr);
}
static int evict(int8_t* k_out, int32_t* kept, int batch, int kv_len, int out_len, int keep, int recent) {
    return slim_cache_evict_int8(by(0), fl(1), by(2), fl(3), fl(4), in(5), k_out, fl(7), by(8), fl(9), fl(10), kept, in(12), batch, 8, kv_len, out_len,
                                 128, keep, recent, nullptr);
}

int main() {
    const int huge = std::numeric_limits<int>::max();
    const int64_t far = std::numeric_limits<int64_t>::max();
    const double nan = std::numeric_limits<double>::quiet_NaN();
    expect(rotate(1024, 1, 4, 128, 16, 0, 1e-6, nullptr), SLIM_ERR_NULL, "rotate null");
    expect(rotate(1016, 1, 4, 128, 16, 0, 1e-6, at(5)), SLIM_ERR_SHAPE, "rotate a stride below a row");
    expect(rotate(far, 1, 4, 128, 16, 0, 1e-6, at(5)), SLIM_ERR_SHAPE, "rotate the largest stride");
    expect(rotate(-far, 1, 4, 128, 16, 0, 1e-6, at(5)), SLIM_ERR_SHAPE, "rotate a negative stride");
    expect(rotate(1028, 1, 4, 128, 16, 0, 1e-6, at(5)), SLIM_ERR_ALIGN, "rotate an odd stride");
    expect(rotate(1024, huge, huge, 128, 16, 0, 1e-6, at(5)), SLIM_ERR_SHAPE, "rotate overflowing sizes");
    expect(rotate(1024, 1, 4, 96, 16, 0, 1e-6, at(5)), SLIM_ERR_UNSUPPORTED, "rotate head_dim");
    expect(rotate(1024, 1, 4, 128, 0, 0, 1e-6, at(5)), SLIM_ERR_SHAPE, "rotate no table");
    expect(rotate(1024, 1, 4, 128, 16, 2, 1e-6, at(5)), SLIM_ERR_SHAPE, "rotate pairs");
    expect(rotate(1024, 1, 4, 128, 16, 0, nan, at(5)), SLIM_ERR_SHAPE, "rotate eps");
    expect(rotate(1024, 1, 4, 128, huge, 0, 1e-6, at(0, 16)), SLIM_ERR_OVERLAP, "rotate into its input");
    expect(rotate(2147483640, 1, 4, 128, 16, 0, 1e-6, at(0, 16)), SLIM_ERR_OVERLAP, "rotate into its input, far rows");
    expect(append(0, in(7), fl(12)), SLIM_ERR_SHAPE, "append empty cache");
    expect(append(64, in(7, 2), fl(12)), SLIM_ERR_ALIGN, "append slots");
    expect(append(64, in(7), fl(12, 4)), SLIM_ERR_ALIGN, "append scales");
    expect(append(64, in(7), fl(10, 64 * 16 * 4 - 16)), SLIM_ERR_OVERLAP, "append scales that meet");
    expect(append(64, nullptr, fl(12)), SLIM_ERR_NULL, "append null slots");

    const size_t p_need = slim_attn_decode_int8_shared_prefix_workspace_bytes(20, 64, 8, 9000, 700, 128);
    if (p_need == 0 || p_need % ((128 + 2) * 4) != 0) { std::fprintf(stderr, "prefix workspace size\n"); ++bad; }
    if (slim_attn_decode_int8_shared_prefix_workspace_bytes(huge, 64, 8, huge, huge, 128) != 0) { std::fprintf(stderr, "prefix workspace, huge\n"); ++bad; }
    expect(prefix(p_need - 1, 20, 9000, 700, 0.1f, at(10)), SLIM_ERR_WORKSPACE, "prefix workspace");
    expect(prefix(p_need, 20, 9000, 700, static_cast<float>(nan), at(10)), SLIM_ERR_SHAPE, "prefix scale");
    expect(prefix(p_need, 20, 0, 700, 0.1f, at(10)), SLIM_ERR_SHAPE, "prefix empty");
    expect(prefix(p_need, huge, 9000, huge, 0.1f, at(10)), SLIM_ERR_SHAPE, "prefix overflowing sizes");
    expect(prefix(p_need, 20, 9000, 700, 0.1f, at(10, 8)), SLIM_ERR_ALIGN, "prefix align");
    expect(prefix(p_need, 20, 9000, 700, 0.1f, nullptr), SLIM_ERR_NULL, "prefix null");
    expect(prefix(p_need, 20, 9000, 700, 0.1f, at(11, 16)), SLIM_ERR_OVERLAP, "prefix into its workspace");
    expect(prefix(p_need, 20, 9000, 700, 0.1f, at(9, 64)), SLIM_ERR_OVERLAP, "prefix over the lengths");
    expect(prefix(p_need, 20, 9000, 700, 0.1f, at(8, -32)), SLIM_ERR_OVERLAP, "prefix over the scales");

    const size_t w_need = slim_attn_decode_int8_weights_workspace_bytes(3, 64, 8, 5000, 128);
    if (w_need < (size_t)3 * 64 * 5000 * 4) { std::fprintf(stderr, "weights workspace size\n"); ++bad; }
    if (slim_attn_decode_int8_weights_workspace_bytes(3, 60, 8, 5000, 128) != 0) { std::fprintf(stderr, "weights workspace of a bad shape\n"); ++bad; }
    expect(weights(w_need - 1, 3, 5000, nullptr, fl(7)), SLIM_ERR_WORKSPACE, "weights workspace");
    expect(weights(w_need, 3, 5000, nullptr, nullptr), SLIM_ERR_NULL, "weights null");
    expect(weights(w_need, 3, 5000, fl(6, 4), fl(7)), SLIM_ERR_ALIGN, "weights align");
    expect(weights(w_need, 3, 5000, fl(7, 16), fl(7)), SLIM_ERR_OVERLAP, "weights that half meet");
    expect(weights(w_need, 3, 5000, nullptr, fl(2, 16)), SLIM_ERR_OVERLAP, "weights over the scales");
    expect(weights(w_need, huge, huge, nullptr, fl(7)), SLIM_ERR_SHAPE, "weights overflowing sizes");

    expect(evict(by(6), in(11), 2, 5000, 700, 0, 0), SLIM_ERR_SHAPE, "evict all");
    expect(evict(by(6), in(11), 2, 5000, 700, 701, 0), SLIM_ERR_SHAPE, "evict to more than there is room for");
    expect(evict(by(6), in(11), 2, 5000, 700, 700, 701), SLIM_ERR_SHAPE, "evict recent");
    expect(evict(by(6), in(11), huge, huge, huge, 700, 1), SLIM_ERR_SHAPE, "evict overflowing sizes");
    expect(evict(by(0, 1024), in(11), 2, 5000, 700, 700, 1), SLIM_ERR_OVERLAP, "evict in place");
    expect(evict(by(6), in(11, 2), 2, 5000, 700, 700, 1), SLIM_ERR_ALIGN, "evict align");
    expect(evict(by(6), nullptr, 2, 5000, 700, 700, 1), SLIM_ERR_NULL, "evict null");
    if (bad == 0) std::printf("serving_abi_sanitize_driver: clean\n");
    return bad ? 1 : 0;
}
