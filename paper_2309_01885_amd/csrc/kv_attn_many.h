// Body of kv_many_kernel and kv_many_mode_kernel (kv_attn.h); DP, GROUP, NT, PARTS and MODE are theirs.
    using R = KvRec<DP, GROUP>;
    using T = KvTiles<DP, GROUP>;
    constexpr int NC = T::NC, NG = T::NG, UT = T::UT, CL = T::CL;
    constexpr int KR = kv_stage_records(DP), W = kKvWaves / KR;  // records of a stage, waves that convert one
    // Records whose exponentials are taken together: all of a stage, where the registers hold them.  Two tiles
    // of two groups spill (2048 queries of 32 heads of 128 in groups of 64 over 8192 tokens: 547 us
    // together, 450 one by one; 96 channels over 4096 226 / 228; groups of 128 over 16384 696 / 737, 64
    // channels in groups of 64 over 8192 273 / 296).
    constexpr int KW = NG == 2 && NT == 2 && DP > 64 ? 1 : KR;
    constexpr int CW = KR == 2 ? NC : (NC + 1) / 2;              // key products a wave converts
    constexpr int VW = T::kHalf ? (UT + 1) / 2 : UT, VK = KR;    // unit tiles and classes
    constexpr int SW = KR == 2 ? (NG + 1) / 2 : (NG + 3) / 4;    // scales a lane converts
    constexpr int SG = SW * (KR == 2 ? 2 : 4);
    struct Stage {
        f16x8 k[KR][2][NC][64], v[KR][UT][CL][64];
        float ks[KR][SG][kKvTok], vs[KR][SG][kKvTok];            // (groups past NG: what lanes without a group write)
        int at[KR];                                              // the records' first tokens
    };
    __shared__ Stage stage[2];
    // workgroups of an XCD (every eighth) get a contiguous stretch of units: rows of the same keys
    // share its L2
    const uint32_t wg = blockIdx.x, q8 = gridDim.x / 8, r8 = gridDim.x % 8, x8 = wg & 7;
    const uint32_t unit = x8 * q8 + min(x8, r8) + (wg >> 3);     // (kKvListed: kv_listed does the same)
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int i = tid & 15, j = lane >> 4;
    KvUnit u;
    if constexpr (MODE == kKvListed) {
        if (!kv_listed(plan, u)) return;
    } else {
        u = kv_unit<MODE>(a, plan, unit, tid == 0);
        if (u.tile_row >= u.rows) return;
    }
    const int r0 = u.rec0, r1 = u.rec1;
    const int row0 = u.tile_row + wave * (16 * NT);

    // what the wave converts: of record `part` of a stage, key half kh from channel block kc on, value
    // classes vk .. of the unit tiles vt, vt + 2, .. (groups of 32) or all
    const int part = wave / W, q = wave % W;
    const int kh = q & 1, kc = KR == 2 ? 0 : (q >> 1) * CW;
    const int vk = T::kHalf ? (KR == 2 ? 0 : q & 1) : KR == 2 ? 2 * (q & 1) : q;
    const int vt = T::kHalf ? (KR == 2 ? q & 1 : q >> 1) : 0;
    const KvBits bits;
    const uint32_t vmask = vk & 1 ? bits.high : bits.low, vshift = vk & 1 ? 4 : 0;   // (KR == 1)
    const int token = T::key_token(i, kh);
    constexpr int VG = T::kHalf ? VW : NG;                       // value groups whose zero points the wave needs
    uint32_t k[CW], kz[CW], v[VW][4], vw[VG][8], word[SW];

    const int64_t pages = a.c.pages_count;
    const int32_t* table = a.table + u.b * a.width;
    const int per = (int)a.c.per;
    // the wave's record of the next stage to be loaded, its page's place in the table and its place in the page
    int next = max(0, min(r0 + part, r1 - 1)), pg = (uint32_t)kv_place<MODE>(u, next) / (uint32_t)per, rem = kv_place<MODE>(u, next) - pg * per;
    int id = r0 < r1 ? table[pg] : 0;
    bool here = false;                                           // whether the record is there (else any other is read, and not used)
    // Starts the loads of the wave's share of the next stage, whose page number was read before, and reads
    // the one after it.  Past the last record it is loaded again.
    auto start = [&] {
        int page = __builtin_amdgcn_readfirstlane(id);
        here = page >= 0 && page < pages;
        if (!here) {
            if (lane == 0) set_status(a.status, QE_ERR_ARG);
            page = 0;
        }
        const uint8_t* rec = a.c.pages + (((int64_t)page * a.c.heads + u.kvh) * per + rem) * R::kBytes;
        kv_words<CW>(rec + (uint32_t)(token * R::kKeyRow + j * (4 * NC)) + 4 * kc, k);
#pragma unroll
        for (int x = 0; x < CW; ++x)
            kz[x] = *reinterpret_cast<const uint32_t*>(rec + (uint32_t)(R::kKeyWords + min((kc + x) / T::CPG, NG - 1) * (4 * kKvTok) + 4 * token));
#pragma unroll
        for (int x = 0; x < VG; ++x)
            kv_words<8>(rec + (uint32_t)(R::kValWords + (T::kHalf ? min(vt + 2 * x, NG - 1) : x) * (4 * kKvTok) + 32 * j), vw[x]);
#pragma unroll
        for (int x = 0; x < VW; ++x)
            kv_words<4>(rec + (uint32_t)(R::kVal + T::unit(T::kHalf ? min(vt + 2 * x, UT - 1) : x, i) * (2 * kKvTok) + 16 * j), v[x]);
#pragma unroll
        for (int x = 0; x < SW; ++x) {
            const bool key = KR == 2 ? kh == 0 : lane < 32;
            const int g = KR == 2 ? min((lane >> 5) + 2 * x, NG - 1) : min(q + 4 * x, NG - 1);
            word[x] = *reinterpret_cast<const uint32_t*>(rec + (uint32_t)((key ? R::kKeyWords : R::kValWords) + g * (4 * kKvTok) + 4 * (lane & 31)));
        }
        const int step = min(KR, r1 - 1 - next);
        if (MODE == kKvSinks && next < u.gap && next + step >= u.gap) {
            const int to = kv_place<MODE>(u, next + step);
            pg = (uint32_t)to / (uint32_t)per;
            rem = to - pg * per;
        } else {
            rem += step;
            while (rem >= per) {
                rem -= per;
                ++pg;
            }
        }
        next += step;
        id = table[pg];                                   // (in a vector register until it is needed: a wait for it now would be one for all loads)
    };
    // r: the first record of the stage
    auto convert = [&](Stage& st, int r) {
#pragma unroll
        for (int x = 0; x < CW; ++x) {
            if (KR == 1 && NC % 2 != 0 && kc + x >= NC) continue;
            uint32_t lo, hi;
            kv_key_zero(kz[x], lo, hi, bits);
            st.k[part][kh][kc + x][lane] = kv_key_frag(k[x], lo, hi, bits);
        }
#pragma unroll
        for (int x = 0; x < VW; ++x) {
            const int t = T::kHalf ? vt + 2 * x : x;
            if (T::kHalf && UT % 2 != 0 && t >= UT) continue;
            uint32_t f[VK][4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t w0 = vw[T::kHalf ? x : T::group_of(x)][2 * p], w1 = vw[T::kHalf ? x : T::group_of(x)][2 * p + 1];
                const uint32_t w = v[x][p] >> (T::kHalf ? i & 8 : vk & 2 ? 8 : 0);
                if constexpr (KR == 2) {
                    uint32_t lo, hi;
                    kv_value_zero(w0, w1, lo, hi, bits);
                    f[0][p] = kv_code_pair(w, bits.low, lo, bits);
                    f[1][p] = kv_code_pair(w, bits.high, hi, bits);
                } else {
                    const uint32_t z = ((__builtin_amdgcn_perm(w1, w0, 0x05040100u) << vshift) & vmask) | bits.z;
                    f[0][p] = kv_code_pair(w, vmask, z, bits);
                }
            }
#pragma unroll
            for (int y = 0; y < VK; ++y) st.v[part][t][vk + y][lane] = kv_frag(f[y][0], f[y][1], f[y][2], f[y][3]);
        }
#pragma unroll
        for (int x = 0; x < SW; ++x) {
            const bool key = KR == 2 ? kh == 0 : lane < 32;
            const int g = KR == 2 ? (lane >> 5) + 2 * x : q + 4 * x;
            float sc = kv_scale(word[x]);
            // (words past the sequence's end, or of a record that is not there, are anything: no scale of theirs may meet a 0)
            sc = !key && (!here || kv_place<MODE>(u, r + part) * kKvTok + (lane & 31) >= u.len) ? 0.f : sc;
            (key ? st.ks : st.vs)[part][g][lane & 31] = sc;
        }
        // (past the last record, or on a page that is not there: past every sequence's end)
        st.at[part] = here && r + part < r1 ? kv_place<MODE>(u, r + part) * kKvTok : 0x7fffff00;
    };

    if (r0 < r1) start();
    KvRows<NC, NT, PARTS, MODE> rows;
    rows.load(a, u, min(row0, u.rows - 1));
    KvSums<T, NT> sums;
    sums.clear();
    if (r0 < r1) {
        convert(stage[0], r0);
        start();
    }
    __syncthreads();
    for (int r = r0, b = 0; r < r1; r += KR, b ^= 1) {
        convert(stage[b ^ 1], r + KR);
        const Stage& st = stage[b];
#pragma unroll
        for (int y0 = 0; y0 < KR; y0 += KW) {
            float s[KW][NT][8];
            int t0[KW];
            bool masked = false;
#pragma unroll
            for (int y = 0; y < KW; ++y) {
                t0[y] = __builtin_amdgcn_readfirstlane(st.at[y0 + y]);
                masked = masked || rows.masked(t0[y]);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    f32x4 acc[NT][2];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) acc[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = g * T::CPG; c < (g + 1) * T::CPG && c < NC; ++c)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const f16x8 f = st.k[y0 + y][h][c][lane];
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int p = 0; p < PARTS; ++p) acc[n][h] = kv_mfma(f, rows.q[p][n][c], acc[n][h]);
                        }
                    const f32x4 s0 = *reinterpret_cast<const f32x4*>(&st.ks[y0 + y][g][8 * j]), s1 = *reinterpret_cast<const f32x4*>(&st.ks[y0 + y][g][8 * j + 4]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float sc = e < 4 ? s0[e] : s1[e - 4], x = acc[n][e >> 2][e & 3];
                            s[y][n][e] = g == 0 ? sc * x : fmaf(sc, x, s[y][n][e]);
                        }
                }
            }
            if (y0 == 0) start();
            KvScales<KW, NG> sv;
            sv.load([&](int y, int g) { return &st.vs[y0 + y][g][8 * j]; });
            sums.template weigh<KW>(s, rows, a.slopes != nullptr, t0, masked, [&](int y, int g, float (&x)[8]) { sv.get(y, g, x); }, [&] { sv.clear(); });
#pragma unroll
            for (int y = 0; y < KW; ++y)
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    f16x8 pr[PARTS][NT];
                    float x[8];
                    sv.get(y, g, x);
                    sums.template weights<PARTS>(s[y], g, x, pr);
#pragma unroll
                    for (int t = 0; t < UT; ++t) {
                        if (T::group_of(t) != g) continue;
#pragma unroll
                        for (int c = 0; c < CL; ++c) {
                            const f16x8 f = st.v[y0 + y][t][c][lane];
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int p = 0; p < PARTS; ++p) sums.o[t][c][n] = kv_mfma(f, pr[p][n], sums.o[t][c][n]);
                        }
                    }
                }
        }
        sums.pin();
        __syncthreads();
    }
    if (row0 >= u.rows) return;
    sums.finish();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 16 * n + i, qi = row / u.per, head = u.kvh * u.per + row - qi * u.per;
        if constexpr (MODE == kKvListed) {
            const int64_t slot = (int64_t)u.slot + (row - u.tile_row);
            sums.octets(n, 0.f, sums.mass[n] == 0.f ? 0.f : 1.f / sums.mass[n], [&](int d, const float* x) {
                if (row >= u.rows) return;
#pragma unroll
                for (int y = 0; y < 8; y += 4) *reinterpret_cast<f32x4*>(plan.part + slot * DP + d + y) = f32x4{x[y], x[y + 1], x[y + 2], x[y + 3]};
            });
            if (row < u.rows && j == 0) {
                const int e = (int)(__float_as_uint(sums.mass[n]) >> 23) - 127;
                plan.stat[2 * slot] = sums.top[n] + (float)e;
                plan.stat[2 * slot + 1] = sums.mass[n] * __uint_as_float((uint32_t)(127 - kKvJoinLog2 - e) << 23);
            }
            continue;
        }
        sums.octets(n, 0.f, sums.mass[n] == 0.f ? 0.f : 1.f / sums.mass[n], [&](int d, const float* x) {
            if (row < u.rows && d < a.c.dim) kv_out8<PARTS>(a, (u.first + qi) * a.ot + head * a.oh + d, x);
        });
        if (row < u.rows && j == 0 && a.lse) a.lse[(u.first + qi) * a.heads + head] = kv_lse(sums.top[n], sums.mass[n]);
    }
