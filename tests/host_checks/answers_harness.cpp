// The argument checks of the calls of a step on a model's own answers (bns_step_validate.hpp, plain C++) under the sanitizers: every combination of extreme
// values in their descriptions, and the overlap tests against what they mean, byte by byte, for small tensors.
#include <stdio.h>

#include <vector>

#include "../../paper_1810_10962_amd/csrc/bns_step_validate.hpp"

using namespace bns;

static int64_t accepted = 0, rejected = 0;

static bns_status count(bns_status s) {
    ++(s == BNS_OK ? accepted : rejected);
    return s;
}

static void extremes() {
    const int64_t rows[] = {INT64_MIN, -1, 0, 1, 7, (int64_t(1) << 31) - 1, int64_t(1) << 31, INT64_MAX};
    const int64_t strides[] = {INT64_MIN, -1, 0, 1, 64, 1001, int64_t(1) << 31, (int64_t(1) << 48) - 1, int64_t(1) << 48, INT64_MAX};
    const int32_t sizes[] = {INT32_MIN, -1, 0, 1, 2, 64, 511, 512, 513, (1 << 20) - 1, 1 << 20, (1 << 30) - 1, 1 << 30, INT32_MAX};
    const float reals[] = {-1.f, -0.f, 0.f, 1e-7f, 1e-6f, 1.f, 1e6f, 1e7f, __builtin_inff(), __builtin_nanf("")};
    for (int64_t t : rows)
        for (int64_t a : strides)
            for (int64_t b : strides)
                for (int32_t h : sizes)
                    for (int32_t w : sizes) {
                        const bns_qk q = {t, {a, b}, {0, 0}, {b, a}, {0, 0}, {0, 0}, {a, 0}, h, 3, w, w & ~1, w & 1, 0, 1, 1e-6f};
                        QkDims d;
                        if (count(check_qk(&q, &d)) != BNS_OK || t == 0 || h == 0) continue;
                        const HeadStrides all[6] = {d.x[0], d.x[1], d.out[0], d.out[1], d.dx[0], d.dx[1]};
                        for (int i = 0; i < 6; ++i) {
                            const __int128 reach = static_cast<__int128>(t - 1) * all[i].token + static_cast<__int128>(d.heads[i % 2] - 1) * all[i].head + w;
                            if (all[i].token < 0 || all[i].head < 0 || reach >= kMostReach) __builtin_trap();
                        }
                        const HeadMatrix m = head_matrix(&d, t, h, w, d.x[0], 4);
                        if (m.m.bytes < size_t(w) * 4 || m.row < size_t(w) * 4) __builtin_trap();
                    }
    for (int64_t t : rows)
        for (int64_t a : strides)
            for (int32_t v : sizes)
                for (int32_t k : sizes)
                    for (int32_t e : {-1, 0, 1, 2})
                        for (float f : reals) {
                            const bns_logprob l = {t, a, 0, v, k, e, f};
                            LogprobDims d;
                            if (count(check_logprob(&l, &d)) == BNS_OK && (d.top > d.vocab || d.logits_stride < d.vocab)) __builtin_trap();
                        }
    for (int64_t n : rows)
        for (int32_t e : {-1, 0, 1, 2})
            for (int32_t r : {0, 1})
                for (uintptr_t p : {uintptr_t(0), uintptr_t(2), uintptr_t(4096)})
                    for (int32_t c : {INT32_MIN, -1, 0, 1, 2, 65537})
                        for (bool scaled : {false, true}) {
                            bns_gradient g[2] = {{reinterpret_cast<void*>(p), reinterpret_cast<void*>(p), n, e, r}, {reinterpret_cast<void*>(1 << 20), nullptr, 0, 0, 0}};
                            if (count(check_gradients(g, c, scaled)) == BNS_OK && scaled) count(gradients_apart(g, c));
                        }
    QkDims q;
    LogprobDims l;
    count(check_qk(nullptr, &q));
    count(check_logprob(nullptr, &l));
    count(check_gradients(nullptr, 1, true));
    printf("accepted %lld rejected %lld\n", static_cast<long long>(accepted), static_cast<long long>(rejected));
}

static char buffer[4096];

static void mark(std::vector<char>& used, int at, int tokens, int heads, int width, const HeadStrides& s) {
    for (int t = 0; t < tokens; ++t)
        for (int h = 0; h < heads; ++h)
            for (int c = 0; c < width; ++c) used[size_t(at + t * s.token + h * s.head + c)] = 1;
}

// Tensors of heads of bytes in one buffer: collide() lets no shared byte pass (except in place), and lets the parts of a projection's result pass.
static void overlaps() {
    long checked = 0, apart = 0;
    const bns_head_strides kinds[] = {{0, 0}, {16, 4}, {20, 3}, {3, 16}, {4, 20}, {24, 0}, {7, 40}};
    for (int tokens = 1; tokens <= 3; ++tokens)
        for (int ha = 1; ha <= 3; ++ha)
            for (int hb = 1; hb <= 3; ++hb)
                for (int width = 1; width <= 3; ++width)
                    for (const bns_head_strides& ka : kinds)
                        for (const bns_head_strides& kb : kinds) {
                            HeadStrides sa, sb;
                            if (head_strides(ka, tokens, ha, width, &sa) != BNS_OK || head_strides(kb, tokens, hb, width, &sb) != BNS_OK) continue;
                            for (int at = -60; at < 60; ++at) {
                                std::vector<char> a(4096, 0), b(4096, 0);
                                mark(a, 1000, tokens, ha, width, sa);
                                mark(b, 1000 + at, tokens, hb, width, sb);
                                bool shared = false;
                                for (size_t i = 0; i < a.size(); ++i) shared |= a[i] && b[i];
                                const HeadMatrix ma = head_matrix(buffer + 1000, tokens, ha, width, sa, 1), mb = head_matrix(buffer + 1000 + at, tokens, hb, width, sb, 1);
                                const bool refused = collide(ma, mb, false);
                                if (shared && !refused) __builtin_trap();
                                if (collide(ma, mb, true) && !refused) __builtin_trap();
                                if (!collide(ma, mb, true) && shared && !(at == 0 && sa.token == sb.token && sa.head == sb.head)) __builtin_trap();
                                apart += !refused;
                                ++checked;
                            }
                        }
    HeadStrides q, k;
    if (head_strides({32, 4}, 5, 4, 4, &q) != BNS_OK || head_strides({32, 4}, 5, 2, 4, &k) != BNS_OK) __builtin_trap();
    if (collide(head_matrix(buffer, 5, 4, 4, q, 1), head_matrix(buffer + 16, 5, 2, 4, k, 1), false)) __builtin_trap();
    // lists of gradients: refused exactly where a result shares a byte with another result or with a gradient that is not its own
    uint32_t seed = 1;
    const auto random = [&](int n) { return int((seed = seed * 1664525u + 1013904223u) >> 8) % n; };
    long lists = 0, fine = 0;
    for (int round = 0; round < 200000; ++round) {
        bns_gradient g[4];
        const int n = 1 + random(4);
        std::vector<int> outs(64, 0), ins(64, 0);
        bool shared = false;
        for (int i = 0; i < n; ++i) {
            const int at = random(20), to = random(3) ? random(20) : at, size = random(5);
            g[i] = {reinterpret_cast<void*>(uintptr_t(4096 + 2 * at)), reinterpret_cast<void*>(uintptr_t(4096 + 2 * to)), size, BNS_BF16, 0};
        }
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j)
                for (int64_t x = 0; x < g[i].elements; ++x)
                    for (int64_t y = 0; y < g[j].elements; ++y) {
                        const auto o = reinterpret_cast<uintptr_t>(g[i].out) + 2 * size_t(x);
                        if (i != j) shared |= o == reinterpret_cast<uintptr_t>(g[j].out) + 2 * size_t(y);
                        if (i != j || g[i].out != g[i].grad) shared |= o == reinterpret_cast<uintptr_t>(g[j].grad) + 2 * size_t(y);
                    }
        if (check_gradients(g, n, true) != BNS_OK) __builtin_trap();
        if ((gradients_apart(g, n) == BNS_OK) == shared) __builtin_trap();
        ++lists;
        fine += !shared;
    }
    printf("checked %ld apart %ld lists %ld fine %ld\n", checked, apart, lists, fine);
}

int main(int argc, char**) {
    if (argc > 1) overlaps();
    else extremes();
    return 0;
}
