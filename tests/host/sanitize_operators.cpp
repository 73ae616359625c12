// Host-only driver for a sanitizer build of the stage executor with rotary positions, norm joins, norms without a mean and distillation: valid and refused layer lists, random
// ones, and passes over plain host memory of exactly the sizes that the library asks for, in which the stand-ins touch all that the kernels would.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "../../include/tmps.h"
#include "operator_stubs.h"

static int bad = 0;
static void expect(bool ok, const char* what) {
    if (!ok) {
        fprintf(stderr, "FAILED: %s (%s)\n", what, tmps_last_error());
        ++bad;
    }
}

static tmps_layer_desc L(int kind, std::initializer_list<int> dims, int flags = 0) {
    tmps_layer_desc d;
    memset(&d, 0, sizeof(d));
    d.kind = kind;
    int i = 0;
    for (int v : dims) d.dims[i++] = v;
    d.flags = flags;
    return d;
}
static int bits(float v) {
    int i;
    memcpy(&i, &v, 4);
    return i;
}
static tmps_stage_cfg cfg(int dtype, int micro, int N, int stash, int last, int borrow) {
    tmps_stage_cfg c;
    c.dtype = dtype; c.micro_batch = micro; c.n_micro = N; c.max_stash = stash; c.is_last = last; c.borrow_input = borrow;
    c.lr = 0.01f; c.momentum = 0.9f;
    return c;
}
static int bytes(const std::vector<tmps_layer_desc>& ls, const tmps_stage_cfg& c, size_t out[4]) {
    return tmps_stage_bytes(ls.data(), (int)ls.size(), &c, &out[0], &out[1], &out[2], &out[3]);
}
static unsigned rnd_state = 777;
static int rnd(int n) {
    rnd_state = rnd_state * 1664525u + 1013904223u;
    return (int)((rnd_state >> 8) % (unsigned)n);
}

// One mini-batch forward and backward on memory that ends where the library says it may.
static void pass(const std::vector<tmps_layer_desc>& ls, int dtype, int micro, int N, int last, int borrow, bool want_dx, int label_ints, int in_place, const char* what) {
    const tmps_stage_cfg c = cfg(dtype, micro, N, 2 * N, last, borrow);
    size_t sz[4];
    expect(bytes(ls, c, sz) == TMPS_OK, what);
    void* p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = aligned_alloc(256, sz[i] ? sz[i] : 256);
        memset(p[i], 0, sz[i] ? sz[i] : 256);
    }
    tmps_stage* st = nullptr;
    expect(tmps_stage_create(&st, ls.data(), (int)ls.size(), &c, p[0], p[1], p[2], p[3]) == TMPS_OK && st, what);
    if (st) {
        const size_t e = dtype == TMPS_F32 ? 4 : 2, in_e = ls[0].kind == TMPS_EMBEDDING ? 4 : e;
        std::vector<char> x((size_t)micro * N * tmps_stage_input_elems(st) * in_e), dy((size_t)micro * N * tmps_stage_output_elems(st) * (last ? 4 : e)), dx(x.size());
        std::vector<int32_t> labels((size_t)micro * N * label_ints + 1);
        std::vector<int> slots;
        for (int round = 0; round < 2; ++round) {
            slots.clear();
            for (int j = 0; j < N; ++j) {
                slots.push_back(N * round + j);
                expect(tmps_forward_micro(st, slots[j], x.data() + j * (x.size() / N), nullptr, last ? labels.data() + (size_t)j * micro * label_ints : nullptr, nullptr, nullptr) == TMPS_OK, what);
            }
            void* out = !want_dx ? nullptr : in_place == 1 ? dy.data() : in_place == 2 ? x.data() : dx.data();
            expect(tmps_backward(st, slots.data(), N, last ? nullptr : dy.data(), out, nullptr) == TMPS_OK, what);
        }
        tmps_stage_destroy(st);
    }
    for (void* q : p) free(q);
}

int main() {
    const int RMS = TMPS_FLAG_RMS, GATE = TMPS_FLAG_GATE;
    const int S = 6, D = 16;
    auto block = [&](int flags) {
        return std::vector<tmps_layer_desc>{L(TMPS_LAYERNORM, {D, S}, flags & RMS), L(TMPS_LINEAR, {D, 3 * D, 0, S}), L(TMPS_ROTARY, {S, D, 2, 1, 3, 0, 2}), L(TMPS_ATTENTION, {S, D, 2}),
                                            L(TMPS_LINEAR, {D, flags & GATE ? 2 * D : D, 0, S}), L(TMPS_NORMJOIN, {D, S, 6}, flags), L(TMPS_LAYERNORM, {D, S}, flags & RMS),
                                            L(TMPS_LINEAR, {D, 24, 0, S}, TMPS_FLAG_GELU), L(TMPS_LINEAR, {24, flags & GATE ? 2 * D : D, 0, S}), L(TMPS_NORMJOIN, {D, S, 4}, flags)};
    };
    for (int dtype : {0, 1})
        for (int flags : {0, RMS, GATE, RMS | GATE})
            for (int borrow : {0, 1})
                for (int dx = 0; dx < 2; ++dx) {
                    operator_stubs = OperatorStubs();
                    pass(block(flags), dtype, 2, 2, 0, borrow, dx, 0, 0, "block");
                    expect(operator_stubs.turned == 4 && operator_stubs.turned_back == 2 && operator_stubs.in_place == 6, "rotary positions are turned where they lie");
                    expect(operator_stubs.joins_with_norm == 4 && operator_stubs.joins == 8 + (flags & RMS ? 4 : 0), "the norm behind a join is in its launch");
                    expect(operator_stubs.joins_back == 4 + (flags & RMS ? 2 : 0), "... in the backward pass as well");
                    std::vector<tmps_layer_desc> student = block(flags);
                    student.insert(student.begin(), L(TMPS_EMBEDDING, {50, S, D}));
                    for (const tmps_layer_desc& l : {L(TMPS_LAYERNORM, {D, S}, RMS), L(TMPS_LINEAR, {D, 50, 0, S}), L(TMPS_DISTILL, {50, S, 4, bits(2.0f), bits(0.5f)})}) student.push_back(l);
                    operator_stubs = OperatorStubs();
                    pass(student, dtype, 3, 2, 1, borrow, false, S * 9, 0, "student");
                    expect(operator_stubs.distillations == 4, "distillation");
                }
    for (int in_place : {1, 2})
        for (int borrow : {0, 1}) pass(block(RMS | GATE), 1, 2, 2, 0, borrow, true, 0, in_place, "dx over an operand");
    pass({L(TMPS_ROTARY, {S, D, 2})}, 1, 2, 2, 0, 1, true, 0, 0, "rotary positions alone");
    pass({L(TMPS_ROTARY, {S, D, 2})}, 1, 2, 2, 0, 0, true, 0, 1, "rotary positions alone, in place");
    pass({L(TMPS_ROTARY, {S, D, 2}), L(TMPS_ATTENTION, {S, D, 2})}, 0, 2, 2, 0, 1, false, 0, 0, "rotary positions first, without an input gradient");
    pass({L(TMPS_LINEAR, {D, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 2}), L(TMPS_LAYERNORM, {D, S}, RMS)}, 1, 2, 3, 0, 0, true, 0, 0, "a norm of the other kind");
    pass({L(TMPS_LINEAR, {D, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 2}), L(TMPS_NORMJOIN, {D, S, 2}), L(TMPS_NORMJOIN, {D, S, 4})}, 1, 2, 2, 0, 0, true, 0, 0, "joins of joins");

    auto refused = [&](std::vector<tmps_layer_desc> ls, tmps_stage_cfg c, int code, const char* what) {
        size_t s4[4];
        expect(bytes(ls, c, s4) == code, what);
    };
    const tmps_stage_cfg c0 = cfg(1, 2, 2, 2, 0, 0), c1 = cfg(1, 2, 2, 2, 1, 0);
    refused({L(TMPS_ROTARY, {S, D, 3})}, c0, TMPS_EINVAL, "heads do not divide the width");
    refused({L(TMPS_ROTARY, {S, 6, 2})}, c0, TMPS_EINVAL, "heads of an odd number of features");
    refused({L(TMPS_ROTARY, {S, D, 2, 0, 0, 3, 2})}, c0, TMPS_EINVAL, "more pairs than a head has");
    refused({L(TMPS_ROTARY, {S, D, 2, -1})}, c0, TMPS_EINVAL, "negative height");
    refused({L(TMPS_ROTARY, {S, D, 2}, TMPS_FLAG_RELU)}, c0, TMPS_EINVAL, "an activation on rotary positions");
    refused({L(TMPS_LINEAR, {4, 3 * D, 0, S}, TMPS_FLAG_RELU), L(TMPS_ROTARY, {S, D, 2})}, c0, TMPS_EUNSUPPORTED, "rotary positions behind an activation");
    refused({L(TMPS_LINEAR, {4, 3 * D, 0, 5}), L(TMPS_ROTARY, {S, D, 2})}, c0, TMPS_ESHAPE, "another number of rows");
    refused({L(TMPS_ROTARY, {1, 1 << 30, 1 << 29})}, c0, TMPS_EUNSUPPORTED, "rows that 32 bits do not count");
    refused({L(TMPS_LINEAR, {D, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 1})}, c0, TMPS_EINVAL, "a join of one source");
    refused({L(TMPS_LINEAR, {D, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 3})}, c0, TMPS_ESHAPE, "a residual before the stage");
    refused({L(TMPS_NORMJOIN, {D, S, 2})}, c0, TMPS_ESHAPE, "a join as the first layer");
    refused({L(TMPS_LINEAR, {8, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 2})}, c0, TMPS_ESHAPE, "a residual of another size");
    refused({L(TMPS_LINEAR, {D, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 2}, GATE)}, c0, TMPS_ESHAPE, "a gate that is not there");
    refused({L(TMPS_LINEAR, {D, D, 0, S}, TMPS_FLAG_GELU), L(TMPS_NORMJOIN, {D, S, 2})}, c0, TMPS_EUNSUPPORTED, "a join behind an activation");
    refused({L(TMPS_LINEAR, {D, D, 0, S}, TMPS_FLAG_RELU), L(TMPS_LINEAR, {D, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 2})}, c0, TMPS_EUNSUPPORTED, "a residual with an activation");
    refused({L(TMPS_LINEAR, {D, D, 0, S}), L(TMPS_NORMJOIN, {D, S, 2}, TMPS_FLAG_RELU)}, c0, TMPS_EINVAL, "an activation on a join");
    refused({L(TMPS_EMBEDDING, {50, S, D}), L(TMPS_NORMJOIN, {D, S, 2})}, c0, TMPS_EUNSUPPORTED, "tokens as a residual");
    refused({L(TMPS_LINEAR, {4, 20000, 0, 1}), L(TMPS_LAYERNORM, {20000, 1}, RMS)}, c0, TMPS_EUNSUPPORTED, "wide rows");
    refused({L(TMPS_LINEAR, {4, 20000, 0, 1}), L(TMPS_LINEAR, {20000, 20000, 0, 1}), L(TMPS_NORMJOIN, {20000, 1, 2})}, c0, TMPS_EUNSUPPORTED, "wide rows of a join");
    refused({L(TMPS_LINEAR, {4, 9, 0, 1}), L(TMPS_DISTILL, {9, 1, 2, bits(1.0f), bits(0.5f)})}, c0, TMPS_ESHAPE, "distillation on a stage that is not the last");
    refused({L(TMPS_LINEAR, {4, 9, 0, 1}), L(TMPS_DISTILL, {9, 1, 0, bits(1.0f), bits(0.5f)})}, c1, TMPS_EINVAL, "no entries");
    refused({L(TMPS_LINEAR, {4, 9, 0, 1}), L(TMPS_DISTILL, {9, 1, 2, bits(0.0f), bits(0.5f)})}, c1, TMPS_EINVAL, "no temperature");
    refused({L(TMPS_LINEAR, {4, 9, 0, 1}), L(TMPS_DISTILL, {9, 1, 2, bits(1.0f), bits(1.5f)})}, c1, TMPS_EINVAL, "alpha above one");
    refused({L(TMPS_LINEAR, {4, 9, 0, 1}), L(TMPS_DISTILL, {9, 1, 2000, bits(1.0f), bits(0.5f)})}, c1, TMPS_EUNSUPPORTED, "too many entries");
    refused({L(TMPS_LINEAR, {4, 9, 0, 3}), L(TMPS_DISTILL, {9, 2, 2, bits(1.0f), bits(0.5f)})}, c1, TMPS_ESHAPE, "another number of rows");
    refused({L(TMPS_LINEAR, {4, 9, 0, 1}, TMPS_FLAG_RELU), L(TMPS_DISTILL, {9, 1, 2, bits(1.0f), bits(0.5f)})}, c1, TMPS_EUNSUPPORTED, "distillation behind an activation");

    // random lists: any answer is fine, reading or writing out of bounds is not
    for (int it = 0; it < 6000; ++it) {
        std::vector<tmps_layer_desc> ls;
        const int kinds[] = {TMPS_LINEAR, TMPS_LINEAR, TMPS_LAYERNORM, TMPS_ROTARY, TMPS_NORMJOIN, TMPS_NORMJOIN, TMPS_ATTENTION, TMPS_DISTILL, TMPS_EMBEDDING};
        const int n = 1 + rnd(7);
        for (int i = 0; i < n; ++i) {
            tmps_layer_desc d;
            memset(&d, 0, sizeof(d));
            d.kind = kinds[rnd(9)];
            for (int k = 0; k < 8; ++k) d.dims[k] = rnd(12) == 0 ? -rnd(3) : rnd(2) ? 4 : rnd(9);
            if (rnd(8) == 0) d.dims[rnd(8)] = rnd(2) ? 2147483647 : 1 << rnd(31);
            d.flags = rnd(3) ? 0 : rnd(64);
            ls.push_back(d);
        }
        size_t s4[4];
        const int N = 1 + rnd(3);
        bool huge = false;   // (sizes whose product is beyond 64 bits are the caller's)
        for (const auto& d : ls)
            for (int v : d.dims) huge = huge || v > (1 << 16);
        if (!huge || ls.size() == 1) (void)bytes(ls, cfg(rnd(2), 1 + rnd(3), N, N * (1 + rnd(2)), rnd(2), rnd(2)), s4);
    }
    return bad ? 1 : 0;
}
