// resq_attend_kv_cache on the host model: cases from standard input, one to a line,
//   B heads_q heads_k d r page order pad window softcap scale missing seed  len ...
// order 0: pages head by head, 1: token by token; pad: bytes behind a row; missing: 1 of so many pages is not there (0: all are).
// Every array is an allocation of its exact size, the last row of the pages at its end, so that the sanitizers see any access beyond
// one.  Prints, per case, how far results are from those of the definition in 64 bits: outputs besides their own rounding, in parts
// of sum_t p_t |v_t|, and log-sum-exps in parts of 1 + |lse|.
#include "resq_kv_api.hip"

#include <iostream>
#include <memory>
#include <random>
#include <sstream>
#include <string>

template <typename T>
struct Exact {   // n elements and not a byte more
    T* p;
    explicit Exact(size_t n, size_t align = 16) {
        void* v;
        if (posix_memalign(&v, align, n * sizeof(T))) abort();
        p = static_cast<T*>(v);
    }
    ~Exact() { free(p); }
    T& operator[](size_t i) { return p[i]; }
};

static uint16_t to_bf16(float x) {
    const uint32_t u = (uint32_t)model::bits(x);
    return (uint16_t)((u + 0x7FFF + (u >> 16 & 1)) >> 16);
}
static double of_bf16(uint16_t x) { return model::real((uint64_t)x << 16); }

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

int main() {
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        int64_t B, hq, hk, d, r, page, order, pad, window, missing, seed;
        double softcap, scale;
        in >> B >> hq >> hk >> d >> r >> page >> order >> pad >> window >> softcap >> scale >> missing >> seed;
        std::mt19937 rng((unsigned)seed);
        auto uniform = [&] { return (float)(rng() >> 8) / (1 << 24); };
        std::vector<int64_t> len(B), held(B);
        int64_t width = 1, total = 0;
        for (int64_t b = 0; b < B; ++b) {
            in >> len[b];
            held[b] = (std::max<int64_t>(len[b], 0) + page - 1) / page;
            width = std::max(width, held[b]);
            total += held[b];
        }
        const int64_t pages = total + 1, RB = r + (d - r) / 2 + 16, rs = order ? hk * (RB + pad) : RB + pad;
        const int64_t hs = order ? RB + pad : page * rs, ps = order ? page * rs : hk * hs;
        Exact<int32_t> lens(B), table(B * width);
        const size_t bytes = (pages - 1) * ps + (hk - 1) * hs + (page - 1) * rs + RB;
        Exact<uint8_t> k(bytes), v(bytes);
        memset(k.p, 255, bytes);   // what no sequence has: codes at their ends, constants NaN
        memset(v.p, 255, bytes);
        std::vector<int32_t> ids(pages);
        for (int64_t i = 0; i < pages; ++i) ids[i] = (int32_t)i;
        std::shuffle(ids.begin(), ids.end(), rng);
        int64_t at = 0;
        for (int64_t b = 0; b < B; ++b) {
            lens[b] = (int32_t)len[b];
            for (int64_t i = 0; i < width; ++i) table[b * width + i] = i < held[b] ? ids[at + i] : -1;
            for (int64_t t = 0; t < len[b]; ++t)
                for (int64_t h = 0; h < hk; ++h)
                    for (uint8_t* base : {k.p, v.p}) {
                        uint8_t* row = base + ids[at + t / page] * ps + h * hs + t % page * rs;
                        for (int64_t i = 0; i < RB - 16; ++i) row[i] = (uint8_t)rng();
                        const float sh = 0.02f * uniform() + 0.005f, sl = 0.2f * uniform() + 0.05f;
                        const float par[4] = {sh, -127 * sh * (1 + 0.1f * uniform()), sl, -7.5f * sl * (1 + 0.1f * uniform())};
                        memcpy(row + RB - 16, par, 16);
                    }
            for (int64_t i = 0; i < held[b]; ++i)
                if (missing && rng() % missing == 0) table[b * width + i] = rng() & 1 ? -1 : (int32_t)pages;
            at += held[b];
        }
        Exact<uint16_t> q(B * hq * d), out(B * hq * d);
        Exact<float> lse(B * hq);
        for (int64_t i = 0; i < B * hq * d; ++i) q[i] = to_bf16(2 * uniform() + 2 * uniform() - 2);
        const size_t need = resq_attend_kv_cache_workspace_bytes(B, hq, hk, d);
        Exact<uint8_t> work(need, 256);
        memset(work.p, 255, need);
        memset(out.p, 255, B * hq * d * 2);
        memset(lse.p, 255, B * hq * 4);
        const int rc = resq_attend_kv_cache(q.p, hq * d, d, B, hq, hk, d, r, lens.p, table.p, width, width, k.p, v.p, pages, page, ps, hs, rs,
                                            (float)scale, (float)softcap, window, out.p, hq * d, d, lse.p, work.p, need, nullptr);
        if (rc) {
            printf("refused %d\n", rc);
            continue;
        }
        double off_out = 0, off_lse = 0;
        for (int64_t b = 0; b < B; ++b)
            for (int64_t h = 0; h < hq; ++h) {
                std::vector<double> x;
                std::vector<Row> rows;
                for (int64_t t = window && len[b] > window ? len[b] - window : 0; t < len[b]; ++t) {
                    const int32_t id = table[b * width + t / page];
                    if (id < 0 || id >= pages) continue;
                    const int64_t where = id * ps + h / (hq / hk) * hs + t % page * rs;
                    const Row key{k.p + where, (int)d, (int)r};
                    rows.push_back(Row{v.p + where, (int)d, (int)r});
                    double s = 0;
                    for (int c = 0; c < d; ++c) s += of_bf16(q[(b * hq + h) * d + c]) * key.value(c, nullptr);
                    s *= scale;
                    x.push_back(softcap > 0 ? softcap * tanh(s / softcap) : s);
                }
                double top = -INFINITY, sum = 0;
                for (double s : x) top = std::max(top, s);
                for (double s : x) sum += exp(s - top);
                const double want_lse = x.empty() ? -INFINITY : top + log(sum), got_lse = lse[b * hq + h];
                if (x.empty() ? got_lse != want_lse : !(fabs(got_lse - want_lse) < INFINITY)) off_lse = INFINITY;
                else if (!x.empty()) off_lse = std::max(off_lse, fabs(got_lse - want_lse) / (1 + fabs(want_lse)));
                for (int c = 0; c < d; ++c) {
                    double want = 0, size = 0;
                    for (size_t i = 0; i < x.size(); ++i) {
                        double one;
                        want += exp(x[i] - want_lse) * rows[i].value(c, &one);
                        size += exp(x[i] - want_lse) * one;
                    }
                    int e;
                    frexp(want, &e);   // |want| in [2^(e-1), 2^e): a step is 2^(e-8)
                    const double off = fabs(of_bf16(out[(b * hq + h) * d + c]) - want) - (want == 0 ? 0 : ldexp(1.0, e - 9));
                    if (!(off < INFINITY)) off_out = INFINITY;
                    else if (off > 0) off_out = std::max(off_out, size ? off / size : INFINITY);
                }
            }
        printf("%.3g %.3g\n", off_out, off_lse);
        fflush(stdout);
    }
}
