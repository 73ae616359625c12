// Host-only driver: the stage executor on launchers that compute (arithmetic.cpp).  Gradients with the one w.r.t. the input written over the upstream gradient or over the borrowed
// input are those of separate arrays, bit for bit; and those of layers that are linear in input and weights are what the outputs change by.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <string>
#include <vector>

#include "../../include/tmps.h"
#include "arithmetic.h"

static int bad = 0;
static void expect(bool ok, const std::string& what) {
    if (!ok) {
        fprintf(stderr, "FAILED: %s (%s)\n", what.c_str(), tmps_last_error());
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
static unsigned rnd_state = 4242;
static int rnd(int n) {
    if (n < 1) return 0;
    rnd_state = rnd_state * 1664525u + 1013904223u;
    return (int)((rnd_state >> 8) % (unsigned)n);
}
static float number() { return (float)(rnd(20001) - 10000) / 10000.0f; }

typedef std::vector<tmps_layer_desc> Layers;
typedef std::vector<float> Numbers;
constexpr int S = 4, D = 8, kMicro = 2, kN = 2;

struct Stage {
    tmps_stage* st = nullptr;
    void* p[4] = {};
    Stage(const Layers& ls, int borrow) {
        const tmps_stage_cfg c = {TMPS_F32, kMicro, kN, kN, 0, borrow, 0.1f, 0.9f};
        size_t sz[4];
        if (tmps_stage_bytes(ls.data(), (int)ls.size(), &c, &sz[0], &sz[1], &sz[2], &sz[3]) != TMPS_OK) return;
        for (int i = 0; i < 4; ++i) {
            p[i] = aligned_alloc(256, (sz[i] + 255) / 256 * 256 + 256);
            memset(p[i], 0, sz[i]);
        }
        tmps_stage_create(&st, ls.data(), (int)ls.size(), &c, p[0], p[1], p[2], p[3]);
    }
    ~Stage() {
        if (st) tmps_stage_destroy(st);
        for (void* q : p) free(q);
    }
    size_t P() const { return (size_t)tmps_stage_param_count(st); }
    size_t in() const { return (size_t)kMicro * kN * tmps_stage_input_elems(st); }
    size_t out() const { return (size_t)kMicro * kN * tmps_stage_output_elems(st); }
    Numbers forward(const Numbers& params, Numbers& x) {
        if (!params.empty()) memcpy(p[0], params.data(), params.size() * 4);
        Numbers y(out());
        for (int j = 0; j < kN; ++j)
            expect(tmps_forward_micro(st, j, x.data() + j * (x.size() / kN), y.data() + j * (y.size() / kN), nullptr, nullptr, nullptr) == TMPS_OK, "forward");
        return y;
    }
    int backward(Numbers& dy, float* dx) {
        const int slots[kN] = {0, 1};
        return tmps_backward(st, slots, kN, dy.data(), dx, nullptr);
    }
    Numbers grads() const { return Numbers((float*)p[1] + P(), (float*)p[1] + 2 * P()); }
};

struct Result {
    int rc = -100;
    Numbers dx, grads;
    bool operator==(const Result& o) const {
        return rc == o.rc && (rc != TMPS_OK || (dx.size() == o.dx.size() && grads.size() == o.grads.size() && !memcmp(dx.data(), o.dx.data(), dx.size() * 4) &&
                                                (grads.empty() || !memcmp(grads.data(), o.grads.data(), grads.size() * 4))));
    }
};
enum Over { kApart, kOverDy, kOverX, kAcrossDy };   // kAcrossDy: from the middle of dy on
static Result run(const Layers& ls, int borrow, Over over, const Numbers& params, const Numbers& x0, const Numbers& dy0) {
    Result r;
    Stage st(ls, borrow);
    if (!st.st) return r;
    Numbers x = x0, dy = dy0, dx(x0.size());
    if (over == kAcrossDy) dy.resize(dy.size() + x0.size());
    st.forward(params, x);
    float* const to = over == kApart ? dx.data() : over == kOverDy ? dy.data() : over == kOverX ? x.data() : dy.data() + dy0.size() / 2;
    r.rc = st.backward(dy, to);
    r.dx.assign(to, to + x0.size());
    r.grads = st.grads();
    return r;
}

static void inputs(const Layers& ls, Numbers& params, Numbers& x, Numbers& dy) {
    Stage st(ls, 0);
    params.clear();
    if (!st.st) return;
    params.resize(st.P());
    x.resize(st.in());
    dy.resize(st.out());
    for (Numbers* v : {&params, &x, &dy})
        for (float& e : *v) e = number();
}

// The same gradients wherever the caller wants the input's.
static bool same(const Layers& ls, const char* what, bool must_pass) {
    Numbers params, x, dy;
    inputs(ls, params, x, dy);
    if (params.empty() && x.empty()) {
        expect(!must_pass, what);
        return false;
    }
    const Result want = run(ls, 1, kApart, params, x, dy);
    expect(!must_pass || want.rc == TMPS_OK, what);
    for (int borrow : {0, 1})
        for (Over over : {kOverDy, kOverX, kAcrossDy}) {
            if (over == kOverDy && dy.size() != x.size()) continue;
            expect(run(ls, borrow, over, params, x, dy) == want, std::string(what) + (over == kOverDy ? ", dx over dy" : over == kOverX ? ", dx over x" : ", dx across the end of dy"));
        }
    return want.rc == TMPS_OK;
}

// Of layers that are linear in x and in every layer's parameters: sum dy (F(x + v) - F(x)) = sum dx v, and the same of each layer's parameters.  Values pass at most 8 layers of sums
// of at most 3 D + 1 terms: off by some 8 * 25 steps of 2^-24 of the sizes that were added up, 1.2e-5; a wrong contribution is off by its own size.
static void differences(const Layers& ls, const char* what) {
    Numbers params, x, dy;
    inputs(ls, params, x, dy);
    const Result got = run(ls, 1, kApart, params, x, dy);
    expect(got.rc == TMPS_OK, what);
    if (got.rc != TMPS_OK) return;
    Stage st(ls, 1);
    const Numbers y = st.forward(params, x);
    expect(st.backward(dy, nullptr) == TMPS_OK, what);
    auto compare = [&](const Numbers& y1, double along, const std::string& which) {
        double change = 0.0, size = 0.0;
        for (size_t i = 0; i < y.size(); ++i) change += (double)dy[i] * ((double)y1[i] - y[i]), size += fabs(dy[i]) * (fabs(y1[i]) + fabs(y[i]));
        expect(fabs(change - along) <= 2e-5 * size + 1e-6, which);
    };
    Numbers x1 = x;
    double along = 0.0;
    for (size_t i = 0; i < x.size(); ++i) {
        const float v = number();
        x1[i] += v;
        along += (double)got.dx[i] * ((double)x1[i] - x[i]);
    }
    compare(st.forward(params, x1), along, std::string(what) + ": dx");
    expect(st.backward(dy, nullptr) == TMPS_OK, what);
    for (size_t li = 0; li < ls.size(); ++li) {
        int64_t at, n, at_b, n_b;
        tmps_stage_param_offset(st.st, (int)li, 0, &at, &n);
        tmps_stage_param_offset(st.st, (int)li, 1, &at_b, &n_b);
        if (!n) continue;
        Numbers p1 = params;
        along = 0.0;
        for (int64_t i = at; i < at + n + n_b; ++i) {
            const float v = number();
            p1[i] += v;
            along += (double)got.grads[i] * ((double)p1[i] - params[i]);
        }
        compare(st.forward(p1, x), along, std::string(what) + ": parameters of layer " + std::to_string(li));
        expect(st.backward(dy, nullptr) == TMPS_OK, what);
    }
}

int main(int argc, char** argv) {
    const std::string which = argc > 1 ? argv[1] : "";
    const tmps_layer_desc dense = L(TMPS_LINEAR, {D, D, 0, S}), wide = L(TMPS_LINEAR, {D, 3 * D, 0, S}), narrow = L(TMPS_LINEAR, {3 * D, D, 0, S}), turned = L(TMPS_ROTARY, {S, D, 2});
    auto join = [](int k, int flags = 0) { return L(TMPS_NORMJOIN, {D, S, k}, flags); };
    auto add = [](int k, int width = D) { return L(TMPS_RESADD, {S, 1, width, k}); };
    for (bool groups : {false, true}) {
        arithmetic.groups = groups;
        if (which == "joins") {
            // residuals that are open when the one from the stage input comes
            for (int open = 0; open <= 9; ++open) {
                Layers ls(10, dense);   // results 0 .. 9
                for (int k = 0; k < open; ++k) ls.push_back(join(10));   // reads the results 0, 1, ...
                ls.push_back(join((int)ls.size() + 1));                  // the stage input
                ls.push_back(dense);
                same(ls, ("a join of the stage input, others open: " + std::to_string(open)).c_str(), true);
            }
            same({dense, join(2), dense, join(4), L(TMPS_LAYERNORM, {D, S}), dense}, "two joins of the stage input", true);
            same({dense, join(2)}, "a join of the stage input alone", true);
        } else if (which == "additions") {
            same({dense, dense, dense, add(4)}, "an addition of the stage input at the end", true);
            same({dense, dense, dense, add(4), dense, dense}, "an addition of the stage input between", true);
            same({dense, add(2), add(3), dense}, "two additions of the stage input", true);
            same({dense, add(2), add(3)}, "two additions of the stage input at the end", true);
            same({L(TMPS_LAYERNORM, {D, S}), dense, add(3), L(TMPS_LAYERNORM, {D, S}), dense, add(3)}, "blocks behind a norm", true);
            Layers ls = {L(TMPS_LAYERNORM, {D, S}), dense, L(TMPS_LINEAR, {D, D, 2, S})};
            same(ls, "a dense layer that adds another's input", true);
        } else if (which == "alone") {
            same({dense}, "one dense layer", true);
            same({L(TMPS_LAYERNORM, {D, S})}, "one norm", true);
            same({L(TMPS_LAYERNORM, {D, S}, TMPS_FLAG_RMS)}, "one norm without a mean", true);
            same({turned}, "rotary positions", true);
            same({dense, dense}, "two dense layers", true);
            // tokens have no gradient: nothing is written
            Numbers params, x, dy;
            const Layers tokens = {L(TMPS_EMBEDDING, {50, S, D})};
            inputs(tokens, params, x, dy);
            const Numbers before(dy.begin(), dy.begin() + (int)x.size());
            const Result r = run(tokens, 1, kOverDy, params, x, dy);
            expect(r.rc == TMPS_OK && r.dx == before, "an embedding alone, dx over dy");
        } else if (which == "rotary") {
            differences({wide, turned, narrow}, "in place");
            differences({turned, narrow}, "first");
            differences({wide, turned, add(2, 3 * D), narrow}, "added to what was turned");
            differences({wide, turned, turned, add(3, 3 * D), narrow}, "added to what was turned twice");
            differences({turned, add(2, 3 * D), narrow}, "added to the stage input");
            differences({turned, turned, add(3, 3 * D), add(3, 3 * D), narrow}, "added, with others, to the stage input");
            differences({wide, turned, narrow, wide, add(4, 3 * D), narrow}, "added to a result that rotary positions read, further up");
            const tmps_layer_desc wide_join = L(TMPS_NORMJOIN, {3 * D, S, 4});
            same({wide, turned, narrow, wide, wide_join}, "joined with a result that rotary positions read", true);
            same({turned, narrow, wide, wide_join}, "joined with the stage input that rotary positions read", true);
        } else if (which == "random") {
            int trained = 0;
            for (int it = 0; it < 4000; ++it) {
                Layers ls;
                const int n = 1 + rnd(10);
                for (int i = 0; i < n; ++i) switch (ls.empty() && rnd(2) ? 0 : rnd(8)) {
                        case 0: ls.push_back(L(TMPS_LAYERNORM, {D, S}, rnd(2) ? TMPS_FLAG_RMS : 0)); break;
                        case 1: case 2: ls.push_back(join(2 + rnd((int)ls.size()), rnd(2) ? TMPS_FLAG_RMS : 0)); break;
                        case 3: case 4: ls.push_back(add(2 + rnd((int)ls.size()))); break;
                        case 5: ls.push_back(wide); ls.push_back(turned); ls.push_back(narrow); break;
                        case 6: ls.push_back(L(TMPS_LINEAR, {D, D, rnd(4) ? 0 : 1 + rnd(3), S})); break;
                        default: ls.push_back(dense);
                    }
                trained += same(ls, "random layers", false);
            }
            expect(trained > 500, "random layers that can be trained");
        } else {
            return 2;
        }
    }
    return bad ? 1 : 0;
}
