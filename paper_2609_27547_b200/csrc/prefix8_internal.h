// Internal declarations of the 8-bit prefix cache operators (include/ebrl_prefix8.h).
#pragma once

#include "../../include/ebrl_prefix8.h"
#include "actgen_internal.h"

#include <atomic>

namespace ebrl {
namespace p8 {

constexpr int BLOCK = 32;          // tokens per scale, per mask word and per tile of the kernels
constexpr int CHUNK_ENVS = 1024;   // environments per launch: their slots and lengths travel as kernel parameters (8 KB)

// A record's parts as byte offsets; everything the kernels need to find a token.
struct Record {
    int kv_layers, kvh, hd, rows, nb;       // rows = capacity rounded up to BLOCK, nb = rows / BLOCK
    size_t plane, scales, mask, bytes;      // bytes of one [rows][hd] plane of one head; offsets of scales and mask; record bytes
    __host__ __device__ size_t head(int layer, int p, int h) const { return (((size_t)layer * 2 + p) * kvh + h) * plane; }
    __host__ __device__ size_t head_scales(int layer, int p, int h) const { return scales + (((size_t)layer * 2 + p) * kvh + h) * nb * 4; }
};
Record record_of(const ebrl_prefix8_layout_t &l);

struct Envs {
    int n;                         // environments of this launch
    int slot[CHUNK_ENVS], len[CHUNK_ENVS];
};

// Attention and weighing: what both take.
struct ReadArgs {
    Record rec;
    const char *pool;
    int layer;
    const void *q;                 // already at the launch's first environment
    long long q_env, q_tok;        // strides in elements
    int H, heads, G;               // G = heads / kv heads: query rows of one kv head are (token, member) pairs, R = H * G of them
    float scale;
    // batches of a handle: records and lengths from the batch's device table instead of pool and Envs
    const EnvMeta *meta;
    int n_envs;
};

struct AttendArgs {
    ReadArgs r;
    int max_len;                   // the longest prefix of the launch
    int alike;                     // whether all are that long
    void *out;
    long long o_env, o_tok;
    float *lse;                    // [env][H][heads] or NULL
    int split, n_split;            // tokens per piece (a multiple of 128), pieces of the longest prefix; 1: not cut
    int team;                      // warps that share an item (one CTA, joined in shared memory); 1 under an SM quota
    float *part_o, *part_ml;       // pieces' results: [env][piece][H * heads][hd], [env][piece][H * heads][2]
    // fp32 models on the tensor cores: the result as three bf16 term planes
    void *out_t1, *out_t2;
    int split_out;
};

struct WeighArgs {
    ReadArgs r;
    const float *lse;
    long long l_env, l_tok, l_head;
    float *weight;                 // row of a slot at weight + slot * stride
    long long stride;
    int accumulate;
};

// attend: query rows (H * G) per item, and items (one warp each) that an SM holds
int attend_tile(int hd, int rows, bool f32, int max_len);
int attend_warps(int hd, int tile);
// grid = CTAs of a persistent grid (an SM quota), 0: as many small CTAs as there are items
cudaError_t launch_attend(const AttendArgs &a, const Envs &e, bool f32, int grid, int sms, cudaStream_t st);
cudaError_t launch_attend_join(const AttendArgs &a, const Envs &e, bool f32, int grid, int n_sms, cudaStream_t st);
cudaError_t launch_weigh(const WeighArgs &a, const Envs &e, bool f32, int max_len, int grid, int sms, cudaStream_t st);

constexpr int QUANT_ENVS = 1024;   // 28 KB of parameters
struct QuantEnvs {
    int n;
    const void *planes[QUANT_ENVS];
    const uint8_t *mask[QUANT_ENVS];
    int slot[QUANT_ENVS], len[QUANT_ENVS], plane_rows[QUANT_ENVS];
};
cudaError_t launch_quantize(const Record &rec, char *pool, long long row_stride, bool f32, const QuantEnvs &e, int max_len, int grid,
                            cudaStream_t st);

constexpr int EVICT_ENVS = 512;
struct EvictEnvs {
    int n;
    int slot[EVICT_ENVS], len[EVICT_ENVS], keep[EVICT_ENVS];   // keep = the new length
};
struct EvictArgs {
    Record rec;
    const char *src;
    char *dst;
    int protect_first, protect_last;
    const float *weight;
    long long weight_stride;
    float *weight_out;
    long long weight_out_stride;
    int *kept;                     // already at the launch's first environment
    long long kept_stride;
};
cudaError_t launch_evict(const EvictArgs &a, const EvictEnvs &e, int max_keep, int grid, int n_sms, cudaStream_t st);

}  // namespace p8
}  // namespace ebrl
