// Drives the page-table work (csrc/pages_ops.h) on the host, under AddressSanitizer and
// UndefinedBehaviorSanitizer without recovery: the calls on consistent tables against their
// definitions written out in order, and on tables and counts of arbitrary words, where
// every access has to stay in bounds.
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include <hip/hip_runtime.h>

#define __hip_atomic_load(p, order, scope) __atomic_load_n(p, order)
inline int atomicMin(int* p, int v) {
    int o = __atomic_load_n(p, __ATOMIC_SEQ_CST);
    while (o > v && !__atomic_compare_exchange_n(p, &o, v, false, __ATOMIC_SEQ_CST, __ATOMIC_SEQ_CST)) {}
    return o;
}
inline int atomicMax(int* p, int v) {
    int o = __atomic_load_n(p, __ATOMIC_SEQ_CST);
    while (o < v && !__atomic_compare_exchange_n(p, &o, v, false, __ATOMIC_SEQ_CST, __ATOMIC_SEQ_CST)) {}
    return o;
}

#include "pages_ops.h"

namespace {

constexpr int NT = 64;
typedef std::vector<int32_t> Words;

uint64_t g_state = 0x9E3779B97F4A7C15ull;
uint64_t next_u64() {  // splitmix64
    uint64_t z = (g_state += 0x9E3779B97F4A7C15ull);
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
int below(int n) { return (int)(next_u64() % (uint64_t)n); }

void expect(bool ok, const char* what) {
    if (!ok) {
        std::fprintf(stderr, "FAILED: %s\n", what);
        std::exit(2);
    }
}

const int kWords[] = {INT_MIN, INT_MIN + 1, -65536, -1, 0, 1, 2, 3, 63, 64, 65, 1000, 4095, 4096, 4097, 65536, 1 << 24,
                      INT_MAX - 4096, INT_MAX - 1, INT_MAX};
int word() {
    if (below(2)) return kWords[below((int)(sizeof(kWords) / sizeof(kWords[0])))];
    return below(3) ? below(300) - 20 : (int)(uint32_t)next_u64();
}

struct Pool {  // a batch's table and the counts of its cache
    int R, maxp, pages, log2P;
    Words table, ref, ctx, want;
    int P() const { return 1 << log2P; }
};

Pool make(bool garbage) {
    Pool p;
    p.R = 1 + below(below(4) ? 12 : 200);
    p.maxp = 1 + below(9);
    p.pages = below(10) ? 1 + below(200) : 4000 + below(5000);
    p.log2P = below(7);
    p.table.assign((size_t)p.R * p.maxp, -1);
    p.ref.assign(p.pages, 0);
    p.ctx.resize(p.R);
    p.want.resize(p.R);
    if (garbage) {
        for (auto* v : {&p.table, &p.ref, &p.ctx, &p.want})
            for (int& x : *v) x = word();
        return p;
    }
    Words ids(p.pages);
    for (int i = 0; i < p.pages; i++) ids[i] = i;
    for (int i = p.pages - 1; i > 0; i--) std::swap(ids[i], ids[below(i + 1)]);
    int used = 0;
    for (int i = 0; i < p.R; i++) {
        p.ctx[i] = below(p.maxp * p.P() + 1);
        const int cols = (p.ctx[i] + p.P() - 1) >> p.log2P, from = i > 0 && below(2) ? below(i) : -1;
        for (int c = 0; c < cols; c++) {
            int pg = from >= 0 && below(4) ? p.table[(size_t)from * p.maxp + c] : -1;  // share some
            if (pg < 0 && used < p.pages && below(10)) pg = ids[used++];
            p.table[(size_t)i * p.maxp + c] = pg;
            if (pg >= 0) p.ref[pg]++;
        }
        p.want[i] = std::min(p.ctx[i] + below(3 * p.P() + 2), p.maxp * p.P());
        if (below(30) == 0) p.want[i] = p.maxp * p.P() + 1;  // more than the table holds
        if (below(10) == 0) p.want[i] = below(p.ctx[i] + 1);
        if (below(60) == 0) p.ctx[i] = -1 - below(5);
    }
    for (; used < p.pages && below(3); used++) p.ref[ids[used]] = 1;  // held by others
    return p;
}

struct Reserved {
    Words table, ref, src, dst, tokens, info;
};

Reserved reserve(const Pool& p, bool alone) {
    Reserved o{p.table, p.ref, Words(p.R, -7), Words(p.R, -7), Words(p.R, -7), Words(4, -7)};
    const int chunks = (p.pages + sv::kPageChunk - 1) / sv::kPageChunk;
    Words writers(p.pages, 99), last(p.pages, 99), demand(p.pages, -5), copy_of(p.pages, -5), upto(p.R), copies(p.R),
        chunk_free(chunks);
    sv::ReserveArgs a{o.table.data(), o.ref.data(), p.ctx.data(), p.want.data(), o.src.data(), o.dst.data(),
                      o.tokens.data(), o.info.data(), p.R, p.maxp, p.pages, p.log2P, chunks, writers.data(),
                      last.data(), demand.data(), copy_of.data(), upto.data(), copies.data(), chunk_free.data(), o.ref.data()};
    auto lds = std::make_unique<sv::ReserveLds<NT>>();
    if (alone) {
        a.was = p.ref.data();
        hosthip::run_workgroup(NT, [&] { sv::reserve_alone<NT>(a, *lds); });
        return o;
    }
    hosthip::run_workgroup(NT, [&] { sv::reserve_demands<NT>(a, *lds); });
    for (int b = 0; b < chunks; b++)
        hosthip::run_workgroup(NT, [&] { sv::count_chunk<NT>(a.ref, a.num_pages, b, false, a.chunk_free, lds->wsum); });
    for (int b = chunks - 1; b >= 0; b--) hosthip::run_workgroup(NT, [&] { sv::reserve_assign<NT>(a, b, lds->wsum); });
    return o;
}

Reserved reserve_in_order(const Pool& p) {
    Reserved o{p.table, p.ref, Words(p.R, -7), Words(p.R, -7), Words(p.R, -7), Words(4, 0)};
    Words free;
    for (int x = 0; x < p.pages; x++)
        if (p.ref[x] == 0) free.push_back(x);
    size_t at = 0;
    for (int i = 0; i < p.R; i++) {
        if (p.ctx[i] < 0) break;
        const int c0 = p.ctx[i] >> p.log2P, c1 = p.want[i] > p.ctx[i] ? (p.want[i] + p.P() - 1) >> p.log2P : c0;
        if (c1 > p.maxp) break;
        Words need;
        for (int c = c0; c < c1; c++) {
            const int pg = o.table[(size_t)i * p.maxp + c];
            if (pg < 0 || o.ref[pg] > 1) need.push_back(c);
        }
        if (need.size() > free.size() - at) break;
        for (int c : need) {
            int& pg = o.table[(size_t)i * p.maxp + c];
            if (pg >= 0) {
                o.ref[pg]--;
                if (c == c0 && (p.ctx[i] & (p.P() - 1))) {
                    o.src[o.info[2]] = pg;
                    o.dst[o.info[2]] = free[at];
                    o.tokens[o.info[2]++] = p.ctx[i] & (p.P() - 1);
                }
            }
            pg = free[at++];
            o.ref[pg] = 1;
        }
        o.info[0]++;
    }
    o.info[1] = (int)at;
    o.info[3] = (int)(free.size() - at);
    return o;
}

void check_reserve(const Pool& p, bool garbage) {
    for (bool alone : {false, true}) {
        const Reserved got = reserve(p, alone);
        if (garbage) continue;
        const Reserved ref = reserve_in_order(p);
        expect(got.info == ref.info, "reserve: info");
        expect(got.table == ref.table && got.ref == ref.ref, "reserve: table and counts");
        expect(got.src == ref.src && got.dst == ref.dst && got.tokens == ref.tokens, "reserve: copies");
    }
}

void check_compact(const Pool& p, bool garbage) {
    const int chunks = (p.pages + sv::kPageChunk - 1) / sv::kPageChunk;
    const int limit = std::min(p.pages / 2, below(2) ? INT_MAX : 1 + below(8));
    Words table = p.table, ref = p.ref, src(limit, -7), dst(limit, -7), info(2, -7), live(chunks), move_of(p.pages, 5);
    sv::CompactArgs a{table.data(), ref.data(), src.data(), dst.data(), info.data(), p.R, p.maxp, p.pages, chunks, limit,
                      live.data(), move_of.data()};
    auto lds = std::make_unique<sv::ReserveLds<NT>>();
    for (int b = 0; b < chunks; b++)
        hosthip::run_workgroup(NT, [&] { sv::count_chunk<NT>(a.ref, a.num_pages, b, true, a.chunk_live, lds->wsum); });
    for (int b = 0; b < chunks; b++) hosthip::run_workgroup(NT, [&] { sv::compact_pair<NT>(a, b, lds->wsum); });
    for (long long e = 0; e < (long long)p.R * p.maxp + limit + 300; e++) sv::compact_entry(a, e);
    if (garbage) return;
    Words t = p.table, r = p.ref, s(limit, -7), d(limit, -7), n(2, 0), to(p.pages);
    for (int x = 0; x < p.pages; x++) n[1] += r[x] > 0, to[x] = x;
    for (int lo = 0, hi = p.pages - 1; n[0] < limit;) {
        while (lo < p.pages && r[lo] > 0) lo++;
        while (hi >= 0 && r[hi] == 0) hi--;
        if (lo >= hi) break;
        s[n[0]] = hi;
        d[n[0]++] = lo;
        std::swap(r[lo], r[hi]);
        to[hi] = lo;
    }
    for (int& x : t)
        if (x >= 0) x = to[x];
    expect(info == n, "compact: info");
    expect(src == s && dst == d, "compact: moves");
    expect(table == t && ref == r, "compact: table and counts");
}

void check_fork(const Pool& p, bool garbage) {
    const int R = 1 + below(20);
    Words parent(R), lens_out(R, -7), out((size_t)R * p.maxp, -7), ref = p.ref;
    for (int& x : parent) x = garbage ? word() : below(p.R + 2) - 1;
    const sv::ForkArgs a{p.table.data(), p.ctx.data(), parent.data(), out.data(), lens_out.data(), ref.data(), R, p.R,
                         p.maxp, p.pages, p.log2P};
    for (long long e = 0; e < ((long long)R + p.R) * p.maxp + 300; e++) sv::fork_entry(a, e);
    if (garbage) return;
    Words r = p.ref;
    for (int x : p.table)
        if (x >= 0) r[x]--;
    for (int i = 0; i < R; i++) {
        const bool ok = parent[i] >= 0 && parent[i] < p.R;
        const int len = ok ? std::max(p.ctx[parent[i]], 0) : 0;
        expect(lens_out[i] == len, "fork: lengths");
        for (int c = 0; c < p.maxp; c++) {
            const int pg = c * p.P() < len ? p.table[(size_t)parent[i] * p.maxp + c] : -1;
            expect(out[(size_t)i * p.maxp + c] == pg, "fork: table");
            if (pg >= 0) r[pg]++;
        }
    }
    expect(ref == r, "fork: counts");
}

void check_release(const Pool& p, bool garbage) {
    const int W = below(2) ? 0 : 1 + below(below(9) ? 200 : INT_MAX), S = below(2) ? 0 : below(below(9) ? 90 : INT_MAX);
    Words table = p.table, ref = p.ref;
    const sv::ReleaseArgs a{table.data(), ref.data(), p.want.data(), p.R, p.maxp, p.pages, p.log2P, W, S};
    for (long long e = 0; e < (long long)p.R * p.maxp + 300; e++) sv::release_entry(a, e);
    if (garbage) return;
    Words r = p.ref;
    for (int i = 0; i < p.R; i++)
        for (int c = 0; c < p.maxp; c++) {
            bool needed = false;  // by a row at position want or later
            for (long long s = (long long)c * p.P(); s < (long long)(c + 1) * p.P(); s++)
                needed |= s < p.want[i] && (W == 0 || s < S || s > (long long)p.want[i] - W);
            const int pg = p.table[(size_t)i * p.maxp + c];
            expect(table[(size_t)i * p.maxp + c] == (needed ? pg : -1), "release: table");
            if (!needed && pg >= 0) r[pg]--;
        }
    expect(ref == r, "release: counts");
}

}  // namespace

int main() {
    int copies = 0, cut = 0;
    for (int n = 0; n < 120; n++) {
        const bool garbage = n % 3 == 2;
        const Pool p = make(garbage);
        check_reserve(p, garbage);
        check_compact(p, garbage);
        check_fork(p, garbage);
        check_release(p, garbage);
        if (!garbage) {
            const Reserved o = reserve_in_order(p);
            copies += o.info[2];
            cut += o.info[0] < p.R;
        }
    }
    expect(copies > 20 && cut > 10, "the cases cover copies and batches that are cut short");
    std::printf("ok: %d copies, %d batches cut short\n", copies, cut);
    return 0;
}
