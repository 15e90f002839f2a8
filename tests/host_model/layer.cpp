// The entry points around a layer's products on the host model: cases from standard input, one to a line,
//   tiles waves B share tokens_q tokens_k  cu_q ... cu_k ...          the search for a workgroup's rows alone
//   prompt hq hk d window softcap scale odd late seed B  new old ...  odd: 1 of so many values is not finite (0: all are)
//   prefix hq hk d r page order pad window softcap scale missing seed prefix B  len ...
//   norm tokens width wide post gate alpha offset eps size pad seed   gate 0: none, 1: one for all tokens, 2: one each
// late: loads straight to LDS arrive when they are waited for, otherwise at once.
// Every array is an allocation of its exact size, so that the sanitizers see any access beyond one.  Prints, per case, how far results
// are from those of the definition in 64 bits: outputs besides their own rounding, in parts of sum_t p_t |v_t| (norm: of themselves),
// and log-sum-exps in parts of 1 + |lse| (norm: the residual sum in parts of its terms).
#include "layer_device.h"

#include "resq_kv_api.hip"
#include "resq_layer_api.hip"

#include <iostream>
#include <random>
#include <sstream>
#include <string>

template <typename T>
struct Exact {   // n elements and not a byte more
    T* p;
    explicit Exact(size_t n, size_t align = 16, int fill = 255) {
        void* v;
        if (posix_memalign(&v, align, n * sizeof(T))) abort();
        memset(v, fill, n * sizeof(T));
        p = static_cast<T*>(v);
    }
    ~Exact() { free(p); }
    T& operator[](size_t i) { return p[i]; }
};

static uint16_t to_bf16(float x) {
    const uint32_t u = (uint32_t)model::bits(x);
    return x != x ? 0x7FC0 : (uint16_t)((u + 0x7FFF + (u >> 16 & 1)) >> 16);
}
static double of_bf16(uint16_t x) { return model::real((uint64_t)x << 16); }

struct Errors {
    double out = 0, sum = 0;
    static void take(double& most, double off) { most = off == off ? std::max(most, off) : INFINITY; }
    // bf16 beside its rounding, in parts of size; what is not finite has to be so on both sides
    void bf16(uint16_t bits, double want, double size) {
        const double got = of_bf16(bits);
        if (!(fabs(want) < INFINITY)) return take(out, got == want || (want != want && got != got) ? 0 : INFINITY);
        int e = 0;
        frexp(want, &e);   // |want| in [2^(e-1), 2^e): half a step is 2^(e-9)
        const double off = fabs(got - want) - (want == 0 ? 0 : ldexp(1.0, e - 9));
        take(out, off > 0 ? size ? off / size : INFINITY : off);
    }
    void lse(float got, double want) { take(sum, want == -INFINITY || want != want ? (got == want || (want != want && got != got) ? 0 : INFINITY) : fabs(got - want) / (1 + fabs(want))); }
};

struct Row {
    const uint8_t* p;
    int d, r;
    double value(int c, double* size) const {
        float par[4];
        memcpy(par, p + r + (d - r) / 2, 16);
        const double s = par[c < r ? 0 : 2], z = par[c < r ? 1 : 3];
        const int code = c < r ? p[c] : p[r + (c - r) / 2] >> (4 * ((c - r) & 1)) & 15;
        if (size) *size = code * s + fabs(z);
        return code * s + z;
    }
};

// one query and head: scores x, values v(i, c, size of it)
template <typename Value>
static void compare(Errors& err, const std::vector<double>& x, int d, Value value, const uint16_t* out, float lse) {
    double top = -INFINITY, sum = 0;
    for (double s : x) top = std::max(top, s);
    for (double s : x) sum += exp(s - top);
    const double want_lse = x.empty() ? -INFINITY : top + log(sum);
    err.lse(lse, want_lse);
    for (int c = 0; c < d; ++c) {
        double want = 0, size = 0;
        for (size_t i = 0; i < x.size(); ++i) {
            double one;
            want += exp(x[i] - want_lse) * value(i, c, &one);
            size += exp(x[i] - want_lse) * fabs(one);
        }
        err.bf16(out[c], want, size);
    }
}
static double capped(double x, double cap) { return cap > 0 ? cap * tanh(x / cap) : x; }

// what prompt_tile finds for each number, by a workgroup as the kernels have them
struct Found {
    int there, last;
    PromptTile tile;
    PromptKeys keys;
};
template <int WAVES>
static void tiles_kernel(const PromptArgs a, Found* found, int first) {
    Found& f = found[blockIdx.x];
    PromptTile tile;
    const bool there = prompt_tile<WAVES>(a, first + (int)blockIdx.x, tile);
    if (threadIdx.x) return;
    f.there = there;
    if (there) {
        f.tile = tile;
        f.keys = prompt_keys<WAVES, 64>(a, tile);
    }
}
// Arrays that do not decrease: each tile once, the last one first.  Any: nothing outside of the tensors.
static void tiles(std::istream& in) {
    int64_t waves, B, share, tokens_q, tokens_k;
    in >> waves >> B >> share >> tokens_q >> tokens_k;
    std::vector<int64_t> got;
    for (int64_t v; in >> v;) got.push_back(v);   // patterns that repeat
    const size_t half = got.size() / 2;
    Exact<int32_t> cu_q(B + 1), cu_k(B + 1);
    bool rises = true;
    for (int64_t b = 0; b <= B; ++b) {
        cu_q[b] = (int32_t)got[b % half];
        cu_k[b] = (int32_t)got[half + b % half];
        rises &= b == 0 || (cu_q[b] >= cu_q[b - 1] && cu_k[b] >= cu_k[b - 1]);
    }
    PromptArgs a{};
    a.cu_q = cu_q.p;
    a.cu_k = cu_k.p;
    a.B = (int)B;
    a.tokens_q = (int)tokens_q;
    a.tokens_k = (int)tokens_k;
    a.share = FastDiv((uint32_t)share);
    a.parts = FastDiv(1u);
    a.window = 1 << 30;
    a.least = 8;
    const int64_t rows = prompt_rows((int)waves), most = (tokens_q * share + B * (rows - 1)) / rows;   // workgroups of a call
    std::vector<int64_t> firsts;
    for (int64_t n = 0; n < most; n += 4)
        if (most <= 64 || n < 16 || n >= most - 16 || n / 4 % (most / 64 + 1) == 0) firsts.push_back(n);
    int64_t wrong = 0, count = 0, at = 0;
    for (int64_t b = 0; b < B; ++b) {
        auto in_range = [&](int64_t x, int64_t n) { return std::min(std::max<int64_t>(x, 0), n); };
        count += (std::max<int64_t>(in_range(cu_q[b + 1], tokens_q) - in_range(cu_q[b], tokens_q), 0) * share + rows - 1) / rows;
    }
    for (int64_t first : firsts) {
        Exact<Found> found(4);
        const auto kernel = waves == 4 ? tiles_kernel<4> : tiles_kernel<8>;
        model::launch([&] { kernel(a, found.p, (int)first); }, dim3(4), dim3(64 * (uint32_t)waves), 0);
        for (int i = 0; i < 4; ++i) {
            const Found& f = found[i];
            if (!f.there) {
                wrong += first + i < std::min(count, most);
                continue;
            }
            const PromptTile& t = f.tile;
            wrong += !(t.q0 >= 0 && t.nq > 0 && (int64_t)t.q0 + t.nq <= tokens_q && t.k0 >= 0 && t.nk >= 0 && (int64_t)t.k0 + t.nk <= tokens_k);
            wrong += !(t.row0 >= 0 && t.row0 < t.rows && t.rows == t.nq * share);
            wrong += !(f.keys.begin >= 0 && f.keys.begin <= f.keys.end && f.keys.end <= t.nk && f.keys.parts >= 1);
            if (rises) {   // its place among all tiles is what was asked for
                at = 0;
                for (int64_t b = 0; b < B && cu_q[b] < t.q0; ++b) at += ((int64_t)(cu_q[b + 1] - cu_q[b]) * share + rows - 1) / rows;
                wrong += at + t.row0 / rows != count - 1 - (first + i);
            }
        }
    }
    printf("%lld %lld\n", (long long)wrong, (long long)count);
}

static void prompt(std::istream& in) {
    int64_t hq, hk, d, window, odd, late, seed, B;
    double softcap, scale;
    in >> hq >> hk >> d >> window >> softcap >> scale >> odd >> late >> seed >> B;
    model::late = late != 0;
    std::mt19937 rng((unsigned)seed);
    auto uniform = [&] { return (float)(rng() >> 8) / (1 << 24); };
    Exact<int32_t> cu_q(B + 1), cu_k(B + 1);
    cu_q[0] = cu_k[0] = 0;
    for (int64_t b = 0; b < B; ++b) {
        int64_t n, o;
        in >> n >> o;
        cu_q[b + 1] = cu_q[b] + (int32_t)n;
        cu_k[b + 1] = cu_k[b] + (int32_t)(n + o);
    }
    const int64_t tq = cu_q[B], tk = cu_k[B];
    Exact<uint16_t> q(tq * hq * d), k(tk * hk * d), v(tk * hk * d), out(tq * hq * d);
    Exact<float> lse(tq * hq);
    for (int64_t i = 0; i < tq * hq * d; ++i) q[i] = to_bf16(2 * uniform() + 2 * uniform() - 2);
    for (int64_t i = 0; i < tk * hk * d; ++i) {
        k[i] = to_bf16(2 * uniform() + 2 * uniform() - 2);
        v[i] = to_bf16(2 * uniform() + 2 * uniform() - 2);
        if (odd && rng() % odd == 0) v[i] = (uint16_t[]){0x7F80, 0xFF80, 0x7FC1}[rng() % 3];
    }
    const size_t need = resq_attend_prompts_workspace_bytes(tq, tk, B, hq, hk, d);
    Exact<uint8_t> work(need, 256);
    const int rc = resq_attend_prompts(q.p, hq * d, d, tq, k.p, hk * d, d, v.p, hk * d, d, tk, cu_q.p, cu_k.p, B, hq, hk, d, (float)scale,
                                       (float)softcap, window, out.p, hq * d, d, lse.p, work.p, need, nullptr);
    if (rc) return (void)printf("refused %d\n", rc);
    Errors err;
    for (int64_t b = 0; b < B; ++b)
        for (int64_t i = 0; i < cu_q[b + 1] - cu_q[b]; ++i)
            for (int64_t h = 0; h < hq; ++h) {
                const int64_t own = i + (cu_k[b + 1] - cu_k[b]) - (cu_q[b + 1] - cu_q[b]), at = (cu_q[b] + i) * hq + h;
                const int64_t first = std::max<int64_t>(window ? own - window + 1 : 0, 0);
                std::vector<double> x;
                for (int64_t j = first; j <= own; ++j) {
                    double s = 0;
                    for (int64_t c = 0; c < d; ++c) s += of_bf16(q[at * d + c]) * of_bf16(k[((cu_k[b] + j) * hk + h / (hq / hk)) * d + c]);
                    x.push_back(capped(s * scale, softcap));
                }
                compare(err, x, (int)d, [&](size_t j, int c, double* size) {
                    return *size = of_bf16(v[((cu_k[b] + first + (int64_t)j) * hk + h / (hq / hk)) * d + c]); }, out.p + at * d, lse[at]);
            }
    printf("%.3g %.3g\n", err.out, err.sum);
}

static void prefix(std::istream& in) {
    int64_t hq, hk, d, r, page, order, pad, window, missing, seed, n, B;
    double softcap, scale;
    in >> hq >> hk >> d >> r >> page >> order >> pad >> window >> softcap >> scale >> missing >> seed >> n >> B;
    std::mt19937 rng((unsigned)seed);
    auto uniform = [&] { return (float)(rng() >> 8) / (1 << 24); };
    auto pages_of = [&](int64_t tokens) { return (std::max<int64_t>(tokens, 0) + page - 1) / page; };
    std::vector<int64_t> len(B);
    int64_t width = 1, total = pages_of(n);
    for (int64_t b = 0; b < B; ++b) {
        in >> len[b];
        width = std::max(width, pages_of(len[b]));
        total += pages_of(len[b]);
    }
    const int64_t pages = total + 1, RB = r + (d - r) / 2 + 16, rs = order ? hk * (RB + pad) : RB + pad;
    const int64_t hs = order ? RB + pad : page * rs, ps = order ? page * rs : hk * hs;
    const size_t bytes = (pages - 1) * ps + (hk - 1) * hs + (page - 1) * rs + RB;
    Exact<uint8_t> k(bytes), v(bytes);   // what no sequence has: codes at their ends, constants NaN
    std::vector<int32_t> ids(pages);
    for (int64_t i = 0; i < pages; ++i) ids[i] = (int32_t)i;
    std::shuffle(ids.begin(), ids.end(), rng);
    int64_t at = 0;
    auto fill = [&](int32_t* table, int64_t wide, int64_t tokens) {
        for (int64_t i = 0; i < wide; ++i) table[i] = i < pages_of(tokens) ? ids[at + i] : -1;
        for (int64_t t = 0; t < tokens; ++t)
            for (int64_t h = 0; h < hk; ++h)
                for (uint8_t* base : {k.p, v.p}) {
                    uint8_t* row = base + ids[at + t / page] * ps + h * hs + t % page * rs;
                    for (int64_t i = 0; i < RB - 16; ++i) row[i] = (uint8_t)rng();
                    const float sh = 0.02f * uniform() + 0.005f, sl = 0.2f * uniform() + 0.05f;
                    const float par[4] = {sh, -127 * sh * (1 + 0.1f * uniform()), sl, -7.5f * sl * (1 + 0.1f * uniform())};
                    memcpy(row + RB - 16, par, 16);
                }
        for (int64_t i = 0; i < pages_of(tokens); ++i)
            if (missing && rng() % missing == 0) table[i] = rng() & 1 ? -1 : (int32_t)pages;
        at += pages_of(tokens);
    };
    Exact<int32_t> prefix_len(1), prefix_table(std::max<int64_t>(pages_of(n), 1)), lens(B), table(B * width);
    prefix_len[0] = (int32_t)n;
    fill(prefix_table.p, std::max<int64_t>(pages_of(n), 1), n);
    for (int64_t b = 0; b < B; ++b) {
        lens[b] = (int32_t)len[b];
        fill(table.p + b * width, width, len[b]);
    }
    Exact<uint16_t> q(B * hq * d), out(B * hq * d);
    Exact<float> lse(B * hq);
    for (int64_t i = 0; i < B * hq * d; ++i) q[i] = to_bf16(2 * uniform() + 2 * uniform() - 2);
    const size_t need = resq_attend_kv_prefix_workspace_bytes(B, hq, hk, d);
    Exact<uint8_t> work(need, 256);
    const int rc = resq_attend_kv_prefix(q.p, hq * d, d, B, hq, hk, d, r, prefix_len.p, prefix_table.p, std::max<int64_t>(pages_of(n), 1), lens.p,
                                         table.p, width, width, k.p, v.p, pages, page, ps, hs, rs, (float)scale, (float)softcap, window, out.p,
                                         hq * d, d, lse.p, work.p, need, nullptr);
    if (rc) return (void)printf("refused %d\n", rc);
    Errors err;
    for (int64_t b = 0; b < B; ++b)
        for (int64_t h = 0; h < hq; ++h) {
            std::vector<double> x;
            std::vector<Row> rows;
            const int64_t first = window ? std::max<int64_t>(n + len[b] - window, 0) : 0;
            for (int64_t t = len[b] < 0 ? n + len[b] : first; t < n + len[b]; ++t) {
                const int32_t id = t < n ? prefix_table[t / page] : table[b * width + (t - n) / page];
                if (id < 0 || id >= pages) continue;
                const int64_t where = id * ps + h / (hq / hk) * hs + (t < n ? t : t - n) % page * rs;
                const Row key{k.p + where, (int)d, (int)r};
                rows.push_back(Row{v.p + where, (int)d, (int)r});
                double s = 0;
                for (int c = 0; c < d; ++c) s += of_bf16(q[(b * hq + h) * d + c]) * key.value(c, nullptr);
                x.push_back(capped(s * scale, softcap));
            }
            compare(err, x, (int)d, [&](size_t i, int c, double* size) { return rows[i].value(c, size); }, out.p + (b * hq + h) * d, lse[b * hq + h]);
        }
    printf("%.3g %.3g\n", err.out, err.sum);
}

template <typename H>
static void norm_of(int64_t tokens, int64_t width, bool post, int64_t gate, double alpha, double offset, double eps, double size, int64_t pad,
                    std::mt19937& rng) {
    auto uniform = [&] { return (float)(rng() >> 8) / (1 << 24); };
    const int64_t ld = width + pad;
    const size_t room = (tokens - 1) * ld + width;
    Exact<uint16_t> y(room, 16), g(gate == 2 ? room : width, 16), x(room, 16), w_pre(width, 16), w_post(width, 16);
    Exact<H> h(room, 16), h_out(room, 16);
    auto put = [](H& to, float f) { to = sizeof(H) == 2 ? (H)to_bf16(f) : (H)f; };
    auto get = [](H from) { return sizeof(H) == 2 ? of_bf16((uint16_t)from) : (double)from; };
    for (int64_t t = 0; t < tokens; ++t)
        for (int64_t c = 0; c < width; ++c) {
            y[t * ld + c] = to_bf16((float)size * (2 * uniform() - 1));
            put(h[t * ld + c], (float)size * (6 * uniform() - 3));
            if (gate == 2) g[t * ld + c] = to_bf16(uniform());
        }
    for (int64_t c = 0; c < width; ++c) {
        w_pre[c] = to_bf16(0.5f + uniform());
        w_post[c] = to_bf16(0.5f + uniform());
        if (gate == 1) g[c] = to_bf16(uniform());
    }
    const int rc = resq_norm_residual(y.p, ld, gate ? g.p : nullptr, gate == 2 ? ld : 0, h.p, ld, sizeof(H) == 4, tokens, width, w_pre.p,
                                      post ? w_post.p : nullptr, (float)offset, (float)eps, (float)alpha, h_out.p, ld, x.p, ld, nullptr);
    if (rc) return (void)printf("refused %d\n", rc);
    Errors err;
    std::vector<double> sum(width), part(width);
    for (int64_t t = 0; t < tokens; ++t) {
        double f = 1, mean = 0;
        if (post) {
            for (int64_t c = 0; c < width; ++c) mean += of_bf16(y[t * ld + c]) * of_bf16(y[t * ld + c]) / width;
            f = 1 / sqrt(mean + (float)eps);
        }
        mean = 0;
        for (int64_t c = 0; c < width; ++c) {
            const double a = of_bf16(y[t * ld + c]) * f * (post ? (float)offset + of_bf16(w_post[c]) : 1) * (gate ? of_bf16(g[(gate == 2 ? t * ld : 0) + c]) : 1);
            sum[c] = get(h[t * ld + c]) + (float)alpha * a;
            part[c] = fabs(get(h[t * ld + c])) + fabs((float)alpha * a);
            mean += sum[c] * sum[c] / width;
        }
        const double root = 1 / sqrt(mean + (float)eps);
        for (int64_t c = 0; c < width; ++c) {
            const double want = sum[c] * root * ((float)offset + of_bf16(w_pre[c]));
            err.bf16(x[t * ld + c], want, part[c] * root);
            int e = 0;
            frexp(sum[c], &e);
            const double off = fabs(get(h_out[t * ld + c]) - sum[c]) - (sum[c] == 0 ? 0 : ldexp(1.0, e - (sizeof(H) == 2 ? 9 : 25)));
            Errors::take(err.sum, off > 0 ? off / part[c] : off);
        }
        for (int64_t c = width; c < ld && t + 1 < tokens; ++c) {   // between the rows nothing is written
            const auto untouched = [](const void* p, size_t n) { return std::all_of((const uint8_t*)p, (const uint8_t*)p + n, [](uint8_t b) { return b == 255; }); };
            if (!untouched(&x[t * ld + c], 2) || !untouched(&h_out[t * ld + c], sizeof(H))) err.out = INFINITY;
        }
    }
    printf("%.3g %.3g\n", err.out, err.sum);
}
static void norm(std::istream& in) {
    int64_t tokens, width, wide, post, gate, pad, seed;
    double alpha, offset, eps, size;
    in >> tokens >> width >> wide >> post >> gate >> alpha >> offset >> eps >> size >> pad >> seed;
    std::mt19937 rng((unsigned)seed);
    (wide ? norm_of<float> : norm_of<uint16_t>)(tokens, width, post != 0, gate, alpha, offset, eps, size, pad, rng);
}

int main() {
    std::string line, op;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        in >> op;
        (op == "tiles" ? tiles : op == "prompt" ? prompt : op == "prefix" ? prefix : norm)(in);
        fflush(stdout);
    }
}
