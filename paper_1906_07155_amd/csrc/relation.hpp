// relation.hpp -- argument blocks and launchers of the relation head's kernels, shared by
// the host API (relation_api.hip) and the kernel translation units.
#pragma once

#include "internal.hpp"

namespace rex {

constexpr int kTile = 32;          // keys of one step of the attention, boxes of one page
constexpr int kAttnWaves = 8;      // waves of one attention workgroup
constexpr int kLdsBytes = 160 << 10;
constexpr float kLog2e = 1.4426950408889634f;

// One side's rows: [batch][row][head][channel], strides in bytes.
struct Rows {
    const void *p;
    int64_t sb;
    uint32_t sr, sh;
};

// The bucket rule of box_relation.h on the bits of |r|: m = (bits >> shift) - base + 1,
// clamped to [0, half].
struct BucketRule {
    int32_t nb, half, shift, base;
};

// Sums of a row's weights: `sum` of them, relative to the exponent
// offset * log2 e + rest (in units of log 2).  The two parts of it stay apart, since a large offset
// (of the biases, natural) would swallow the rest, and the rest is binary64 for the sake of large
// products.
struct SumRef {
    float offset, sum;
    double rest;
};

struct AttnArgs {
    Rows q, k, v;
    const float *qbox, *kbox;           // element strides of batch and row below
    int64_t qbox_sb, qbox_sr, kbox_sb, kbox_sr;
    const float *bias;                  // [H][nb * nb] or null
    const int32_t *qlen, *klen;
    const uint8_t *kmask;
    BucketRule rule;
    float scale;                        // of the logits, natural
    int32_t B, Nq, Nk, H, Hkv, D;
    int32_t group;                      // H / Hkv
    // the paged memory (k and v then unused)
    const int8_t *mk, *mv;
    const float *mks, *mvs, *mbox;
    const int32_t *pages;
    int64_t num_pages;
    int32_t max_pages;
    // forward
    void *out;
    float *out_f32, *lse;
    int32_t terms;                      // dense keys: parts of the weights that multiply bf16 data, 2 or 3
    float *part;                        // nsplit > 1: partial sums [nsplit][B][H][Nq][D],
    SumRef *part_ml;                   // and what they refer to [nsplit][B][H][Nq]
    int32_t nsplit;
    // how a workgroup's waves are shared out: heads x parts of the streamed side
    int32_t hp, parts;
    int32_t tiles;                      // column tiles of one image
    int32_t nwg, per;                   // workgroups, and those of them that share keys
    // backward
    Rows gout;                          // grad_out, dense
    const void *fout;                   // what the forward wrote
    const float *fout_f32, *flse;
    void *gq, *gk, *gv;
    float *gbias;
    float *rowstat;                     // [B][H][Nqp][2]: lse in units of log 2 (+inf: no row), delta
    float *rowfar;                      // [B][H][Nqp][2]: of rows with a far lse, what it is relative to
    int32_t *far;                       // [B][H][Nqp / 16]: whether there are such among 16 rows
    float *hist;                        // [B * spans][H][nb * nb]
    int32_t Nqp;
    int32_t span, spans;                // key tiles of one workgroup, runs of them per image
    int32_t head_step;                  // heads of a group whose tables are in LDS together
};

hipError_t launch_attn_fwd(const AttnArgs &a, int dtype, int cols, hipStream_t s);
hipError_t launch_attn_recall(const AttnArgs &a, int dtype, int cols, hipStream_t s);
hipError_t launch_attn_combine(const AttnArgs &a, int dtype, hipStream_t s);
// Whether a workgroup of the key pass with `cols` key columns fits the LDS.
bool dkv_fits(const AttnArgs &dkv, int dtype, int cols);
hipError_t launch_attn_bwd(const AttnArgs &dq, const AttnArgs &dkv, int dtype, int dq_cols,
                           int dkv_cols, hipStream_t s);

struct MemoryArgs {
    int8_t *k8, *v8;
    float *ks, *vs, *mbox;
    int64_t num_slots;
    int32_t Hkv, D;
    const int64_t *slots;
    int64_t count;
    const void *k, *v;                  // append: element strides of row and head
    int64_t k_sr, k_sh, v_sr, v_sh;
    const float *boxes;
    int32_t owned;                      // pages of one workgroup, where those share the work
    int32_t vec;                        // append: rows can be read 16 bytes at a time
    void *k_out, *v_out;                // read
    float *boxes_out;
};

hipError_t launch_memory_append(MemoryArgs a, int dtype, hipStream_t s);
hipError_t launch_memory_read(MemoryArgs a, int dtype, hipStream_t s);

struct NormArgs {
    const void *x, *branch;
    int64_t x_stride, b_stride;
    int64_t rows, rows_per_gate;
    FastDiv gate_div;                   // by rows_per_gate
    int32_t C;
    int32_t layer;
    float alpha, eps;
    const float *gate, *w1, *c1, *w2, *c2;
    void *y, *u;
    float *stats;
    int32_t second;                     // the second norm takes part
    int32_t vec;                        // rows can be read and written 16 bytes at a time
    int32_t pvec;                       // parameters too
    // backward
    const void *gy, *gu;
    void *gx, *gb;
    float *ggate, *gw1, *gc1, *gw2, *gc2;
    float *part;                        // [blocks][4][C]: sums for gw1, gc1, gw2, gc2
    float *gate_part;                   // [gates * gate_parts][C]
    int32_t gate_sum;                   // ggate is the sum of gate_part's rows
    // Forward: unit_rows rows for each of `blocks` workgroups.
    // Backward: a unit is a run of rows of one gate row: unit i holds rows from
    // (i / gate_parts) * span + (i % gate_parts) * unit_rows on, span rows per gate row.
    int64_t units, span, gates;
    int32_t gate_parts, unit_rows, blocks;
};

int norm_slots(int dtype, int C);   // rows a workgroup takes side by side
hipError_t launch_norm_fwd(const NormArgs &a, int dtype, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs &a, int dtype, hipStream_t s);

}  // namespace rex
