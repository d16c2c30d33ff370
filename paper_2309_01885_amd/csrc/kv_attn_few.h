// Body of kv_few_kernel, kv_few_mode_kernel (kv_attn.h) and kv_pair_kernel (kv_attn_modes.h); DP, GROUP, NT, PARTS, MODE
// and lds (a KvFewLds) are theirs.
    using R = KvRec<DP, GROUP>;
    using T = KvTiles<DP, GROUP>;
    constexpr int NC = T::NC, NG = T::NG, UT = T::UT, CL = T::CL;
    const uint32_t unit = MODE == kKvListed ? 0 : blockIdx.x / (uint32_t)plan.nsplit;
    const int split = MODE == kKvListed ? 0 : (int)(blockIdx.x - unit * plan.nsplit);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i = tid & 15, j = (tid & 63) >> 4;
    KvUnit u;
    if constexpr (MODE == kKvListed) {
        if (!kv_listed(plan, u)) return;
    } else {
        u = kv_unit<MODE>(a, plan, unit, tid == 0 && split == 0);
        if (split >= u.splits || u.tile_row >= u.rows) return;
    }
    const int r1 = MODE == kKvListed ? u.rec1 : u.from(split + 1);
    int r = (MODE == kKvListed ? u.rec0 : u.from(split)) + wave;

    // A record's codes, and a word of each group: a key's (lanes 0 .. 31) or a value's.  The keys' registers
    // are free once the scores are there and take the next record's keys; the values' likewise after
    // the weighted sum.  The words' scales and zero points reach the lanes that need them through the
    // wave's part of LDS.  (Read from memory by each of those lanes they took 18 registers a group and
    // 32 more instructions.)
    typename KvFewLds<DP, GROUP, NT>::Words& held = lds.words[wave];
    const int lane = tid & 63;
    const KvBits bits;
    uint32_t k[2][NC], v[UT][4], word[NG];
    const int64_t pages = a.c.pages_count;
    const int32_t* table = a.table + u.b * a.width;
    const int per = (int)a.c.per;
    int pg = (uint32_t)kv_place<MODE>(u, r) / (uint32_t)per, rem = kv_place<MODE>(u, r) - pg * per;
    int id = r < r1 ? table[pg] : 0;
    const uint8_t* rec = a.c.pages;
    bool here = false;                                           // whether the record is there (else any other is read, and not used)
    // The address of record r, whose page number was read before; reads the one after it.
    auto find = [&](int r) {
        int page = __builtin_amdgcn_readfirstlane(id);
        here = page >= 0 && page < pages;
        if (!here) {
            set_status(a.status, QE_ERR_ARG);
            page = 0;
        }
        rec = a.c.pages + (((int64_t)page * a.c.heads + u.kvh) * per + rem) * R::kBytes;
        if (MODE == kKvSinks && r < u.gap && r + kKvWaves >= u.gap) {
            const int to = kv_place<MODE>(u, r + kKvWaves);
            pg = (uint32_t)to / (uint32_t)per;
            rem = to - pg * per;
        } else {
            rem += kKvWaves;
            while (rem >= per) {
                rem -= per;
                ++pg;
            }
        }
        if (r + kKvWaves < r1) id = table[pg];            // (in a vector register until it is needed: a wait for it now would be one for all loads)
    };
    auto keys = [&] {
#pragma unroll
        for (int g = 0; g < NG; ++g)
            word[g] = *reinterpret_cast<const uint32_t*>(rec + (uint32_t)((lane < 32 ? R::kKeyWords : R::kValWords) + g * (4 * kKvTok) + 4 * (lane & 31)));
#pragma unroll
        for (int h = 0; h < 2; ++h) kv_words<NC>(rec + (uint32_t)(T::key_token(i, h) * R::kKeyRow + j * (4 * NC)), k[h]);
    };
    auto values = [&] {
#pragma unroll
        for (int t = 0; t < UT; ++t) kv_words<4>(rec + (uint32_t)(R::kVal + T::unit(t, i) * (2 * kKvTok) + 16 * j), v[t]);
    };
    // (LDS serves a wave in order: what was read before is not overwritten.)
    auto hold = [&](int t0) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            // words past the sequence's end are anything: no value scale of theirs may meet a 0
            held.s[g][lane] = lane >= 32 && t0 > u.len - 1 - (lane & 31) ? 0.f : kv_scale(word[g]);
            held.lo[g][lane] = (uint16_t)(0xE400u | (word[g] & 15u));
            held.hi[g][lane] = (uint16_t)(0xE400u | (word[g] & 15u) << 4);
        }
        __builtin_amdgcn_wave_barrier();
    };
    auto first_token = [&](int r) { return here ? kv_place<MODE>(u, r) * kKvTok : 0x7fffff00; };    // (of no record: past every sequence's end)
    if (r < r1) {
        find(r);
        keys();
        values();
    }
    KvRows<NC, NT, PARTS, MODE> rows;
    rows.load(a, u, u.tile_row);
    KvSums<T, NT> sums;
    sums.clear();

    int t0 = first_token(r);
    if (r < r1) hold(t0);
    for (; r < r1; r += kKvWaves) {
        const bool masked = rows.masked(t0), more = r + kKvWaves < r1;
        const int at[1] = {t0};
        float s[1][NT][8];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f32x4 acc[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t l = held.lo[g][T::key_token(i, h)], x = held.hi[g][T::key_token(i, h)], lo = l << 16 | l, hi = x << 16 | x;
#pragma unroll
                for (int c = g * T::CPG; c < (g + 1) * T::CPG && c < NC; ++c) {
                    const f16x8 f = kv_key_frag(k[h][c], lo, hi, bits);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) acc[n][h] = kv_mfma(f, rows.q[p][n][c], acc[n][h]);
                }
            }
            const f32x4 s0 = *reinterpret_cast<const f32x4*>(&held.s[g][8 * j]), s1 = *reinterpret_cast<const f32x4*>(&held.s[g][8 * j + 4]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float sc = e < 4 ? s0[e] : s1[e - 4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float x = acc[n][e >> 2][e & 3];
                    s[0][n][e] = g == 0 ? sc * x : fmaf(sc, x, s[0][n][e]);
                }
            }
        }
        if (more) {
            find(r + kKvWaves);
            keys();
        }
        KvScales<1, NG> sv;
        sv.load([&](int, int g) { return &held.s[g][32 + 8 * j]; });
        sums.template weigh<1>(s, rows, a.slopes != nullptr, at, masked, [&](int y, int g, float (&x)[8]) { sv.get(y, g, x); }, [&] { sv.clear(); });
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f16x8 pr[PARTS][NT];
            float x[8];
            sv.get(0, g, x);
            sums.template weights<PARTS>(s[0], g, x, pr);
            const u32x4 lo = *reinterpret_cast<const u32x4*>(&held.lo[g][32 + 8 * j]), hi = *reinterpret_cast<const u32x4*>(&held.hi[g][32 + 8 * j]);
#pragma unroll
            for (int t = 0; t < UT; ++t) {
                if (T::group_of(t) != g) continue;
                uint32_t w[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) w[p] = T::kHalf ? v[t][p] >> (i & 8) : v[t][p];
#pragma unroll
                for (int c = 0; c < CL; ++c) {
                    uint32_t pair[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) pair[p] = kv_code_pair(w[p] >> (c >= 2 ? 8 : 0), c & 1 ? bits.high : bits.low, c & 1 ? hi[p] : lo[p], bits);
                    const f16x8 f = kv_frag(pair[0], pair[1], pair[2], pair[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) sums.o[t][c][n] = kv_mfma(f, pr[p][n], sums.o[t][c][n]);
                }
            }
        }
        if (more) {
            values();
            t0 = first_token(r + kKvWaves);
            hold(t0);
        }
        sums.pin();
    }
    sums.finish();

    // every wave to the common maximum, divided by the common mass (sums of large values would pass the
    // largest number before it), then sums over the waves
    auto &wtop = lds.wtop, &wmass = lds.wmass;
    auto &rtop = lds.rtop, &rmass = lds.rmass;
    auto& acc = lds.acc;                                      // (written after a barrier that ends the use of the words)
#pragma unroll
    for (int n = 0; n < NT; ++n)
        if (j == 0) {
            wtop[wave][16 * n + i] = sums.top[n];
            wmass[wave][16 * n + i] = sums.mass[n];
        }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float m = -kKvInf, l = 0.f;
#pragma unroll
        for (int w = 0; w < kKvWaves; ++w) m = fmaxf(m, wtop[w][16 * n + i]);
#pragma unroll
        for (int w = 0; w < kKvWaves; ++w) {
            const float t = wtop[w][16 * n + i];
            l = fmaf(t == m ? 1.f : __builtin_amdgcn_exp2f(t - m), wmass[w][16 * n + i], l);
        }
        if (wave == 0 && j == 0) {
            rtop[16 * n + i] = m;
            rmass[16 * n + i] = l;
        }
        sums.octets(n, m == sums.top[n] ? 0.f : sums.top[n] - m, l == 0.f ? 0.f : 1.f / l, [&](int d, const float* x) {
#pragma unroll
            for (int y = 0; y < 8; y += 4) *reinterpret_cast<f32x4*>(&acc[wave][16 * n + i][d + y]) = f32x4{x[y], x[y + 1], x[y + 2], x[y + 3]};
        });
    }
    __syncthreads();
    for (int x = tid; x < 16 * NT * (DP / 8); x += 256) {
        const int rr = x / (DP / 8), d = 8 * (x - rr * (DP / 8)), row = u.tile_row + rr;
        if (row >= u.rows) break;
        f32x4 sum[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const f32x4 s0 = *reinterpret_cast<const f32x4*>(&acc[0][rr][d + 4 * y]), s1 = *reinterpret_cast<const f32x4*>(&acc[1][rr][d + 4 * y]);
            const f32x4 s2 = *reinterpret_cast<const f32x4*>(&acc[2][rr][d + 4 * y]), s3 = *reinterpret_cast<const f32x4*>(&acc[3][rr][d + 4 * y]);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[y][e] = (s0[e] + s1[e]) + (s2[e] + s3[e]);
        }
        const float m = rtop[rr], l = rmass[rr];
        if (MODE == kKvListed || u.splits > 1) {
            const int64_t slot = MODE == kKvListed ? (int64_t)u.slot + rr : ((int64_t)unit * plan.nsplit + split) * plan.rows + rr;
#pragma unroll
            for (int y = 0; y < 2; ++y) *reinterpret_cast<f32x4*>(plan.part + slot * DP + d + 4 * y) = sum[y];
            if (d == 0) {
                const int e = (int)(__float_as_uint(l) >> 23) - 127;      // (of no mass: m is -inf)
                plan.stat[2 * slot] = m + (float)e;
                plan.stat[2 * slot + 1] = l * __uint_as_float((uint32_t)(127 - kKvJoinLog2 - e) << 23);
            }
        } else {
            const int qi = row / u.per, head = u.kvh * u.per + row - qi * u.per;
            float out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = sum[e >> 2][e & 3];
            if (d < a.c.dim) kv_out8<PARTS>(a, (u.first + qi) * a.ot + head * a.oh + d, out);
            if (a.lse && d == 0) a.lse[(u.first + qi) * a.heads + head] = kv_lse(m, l);
        }
    }
