// What a workgroup does for 128 query columns and a span of tokens: the body of wide_kernel, and of wide_piece where slots share pages.  It is text
// that both include, as the compiler schedules the loop worse in a function that the kernel calls, inlined or not: 4 prompts of 4096 tokens, 40 heads, first
// tokens and a window, 402 us as text, 412 as a call.
//
//   kTrunk            whether it is a piece of the plan's nodes
//   c, a              as everywhere
//   id, items, splits the item of the launch (not kTrunk)
//   trunk             the piece (kTrunk)
//   tiles_of, spoiled in LDS

  constexpr int H = D / 64, KK = D / 16, OB = D / 32;
  auto keys = tiles_of, values = tiles_of + 2;
  const int wave = __builtin_amdgcn_readfirstlane(thread_of<Args>() >> 6), lane = thread_of<Args>() & 63, n = lane & 31, h = lane >> 5;
  const int G = c.q_per_kv;
  const int split = kTrunk ? 0 : id % (unsigned)splits;
  const unsigned item = kTrunk ? 0 : id / (unsigned)splits;
  const int head = kTrunk ? trunk.head : item / items;
  Columns t;
  Rows rows;
  if constexpr (kTrunk) {                            // rows of several slots
    t = Columns{trunk.node.slot, trunk.column, trunk.node.cols, 0};
    rows = Rows{trunk.node.row, trunk.node.rows};
  } else {
    if (!columns_of(c, a, item % items, splits == 1 && c.slots <= kWave, t, rows)) return;
  }
  const int len = t.len, before = len - rows.count;
  const int last_col = min(t.first + kWide, t.count) - 1;
  const int lo = kTrunk ? trunk.node.lo : before + t.first / G, hi = kTrunk ? trunk.node.hi : before + last_col / G;
  const auto span = [&] {
    if constexpr (kTrunk) return Cut(span_of(c, lo, hi), trunk.node.first, trunk.node.last);
    else return span_of(c, lo, hi);
  }();
  const int tiles = (span.count + 3) / 4, each = max(2, (tiles + splits - 1) / splits);
  const int from = kTrunk ? trunk.from : split * each, to = min(tiles, kTrunk ? trunk.to : from + each);

  // this wave's columns
  const int col = t.first + wave * 32 + n;
  const int wave_last = min(t.first + wave * 32 + 31, last_col);
  // (a node's rows have their positions in any order, as the plan has them: what tiles all of them see is known from the least and the largest)
  const int wave_lo = kTrunk ? lo : before + (t.first + wave * 32) / G, wave_hi = kTrunk ? hi : before + wave_last / G;
  const bool have = t.first + wave * 32 <= last_col;
  const int row = rows.first + col / G, q_head = head * G + col % G;
  // the row, at p, sees the tokens from_token .. p and those before first_tokens
  const int p = [&] {
    if constexpr (kTrunk) return col <= last_col ? min(max(a.plan.pos[row], -1), c.table_len * c.page_tokens - 1) : -1;
    else return col <= last_col ? before + col / G : -1;
  }();
  const int from_token = c.window > 0 ? max(max(p, 0) - c.window + 1, 0) : 0, first_tokens = c.window > 0 ? min(c.sinks, p + 1) : 0;
  u4 q[KK];
#pragma unroll
  for (int k = 0; k < KK; ++k) {
    q[k] = u4{0, 0, 0, 0};
    if (col <= last_col) q[k] = reinterpret_cast<const u4 *>(a.q)[row * (a.stride / 8) + q_head * (D / 8) + k * 2 + h];
  }

  // Tiles that all rows of the workgroup, of this wave, see in full: a range [first, last) of the list, none where a page of the
  // slot is missing (which the look-ups below find before such a tile is reached).
  const int all_first = inner_first(c, span, hi), mine_first = inner_first(c, span, wave_hi);
  int all_last = inner_last(span, lo), mine_last = inner_last(span, wave_lo);

  // Blocks are looked up for sixteen tiles at a time, a lane each: the table a chunk ahead, the exponents half a chunk ahead.
  constexpr int kChunk = kWave / 4;
  const int *table = c.table + (size_t)t.slot * c.table_len;
  int chunk = from, page, at, at_next, exps_next;    // at: the lane's block in the pool, -1: not there
  float factor, shift, unit;                         // of the lane's block: t = factor x + shift; its weights add to the sum times unit
  auto look = [&](int tile) {                        // of the chunk that begins with this tile
    const int i = tile * 4 + lane;
    page = table[i < to * 4 && i < span.count ? entry_of(c, span.block(i)) : 0];      // (not looked at here: it is on its way)
  };
  auto place = [&](int tile) {
    const int i = tile * 4 + lane;
    at_next = i < to * 4 && i < span.count ? block_in(c, page, head, span.block(i)) : -1;
    exps_next = reinterpret_cast<const unsigned short *>(c.exps)[max(at_next, 0)];
    if (__ballot(at_next < 0 && i < to * 4 && i < span.count)) all_last = mine_last = 0;
  };
  auto turn = [&] {
    at = at_next;
    const int ex = at < 0 ? 0 : exps_next;           // (of what is not there the load gave any block's: powers of two that are no numbers, perhaps)
    factor = pow2((signed char)ex) * c.scale_log2;
    const int e = (signed char)(ex >> 8);
    shift = (float)e;
    unit = pow2(-e);
  };
  auto at_of = [&](int tile, int b) {
    const int i = tile - chunk;
    return __builtin_amdgcn_readlane(i < kChunk ? at : at_next, i % kChunk * 4 + b);
  };

  // Staging.  A wave brings halves of 64 channels of a block: D = 128 two of them (blocks wave / 2 and wave / 2 + 2), D = 64 one.  Every load
  // is made (of the pool's first block where there is none to read).
  u4 kc[H], vc[H];
  auto piece_block = [&](int j) { return H == 2 ? wave / 2 + 2 * j : wave; };
  const int half = H == 2 ? wave % 2 : 0;
  auto request = [&](int tile) {
    if (tile >= to) return;
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const int block = max(at_of(tile, piece_block(j)), 0);
      const Bytes k = scalar_bytes(c.k, block * ((long)kBlock * D)), v = scalar_bytes(c.v, block * ((long)kBlock * D));
      kc[j] = *(Pieces)(k + (unsigned)(half * kWave + lane) * 16);
      vc[j] = *(Pieces)(v + (unsigned)(half * kWave + lane) * 16);
    }
  };
  // where a word of four tokens' codes of channel 64 half + 16 i + (lane & 15) goes: [block][32 channels][which eight of the 16
  // tokens][channel], tokens 0-3 and 8-11, or 4-7 and 12-15
  auto value_at = [&](int j, int i) {
    const int d = half * 64 + i * 16 + (lane & 15), g = lane >> 4;
    return (((piece_block(j) * OB + d / 32) * 2 + (g & 1)) * 32 + d % 32) * 2 + (g >> 1);
  };
  bool mine_spoiled = false;
  auto stage = [&](int tile, int buf) {
    const int tok = lane & 15, g = lane >> 4;
    // what no row sees is left out, and a NaN among values that only some rows see is taken out (0 * NaN is NaN) and given to those
    // that see it in the end
    if (tile < all_first || tile >= all_last) {
#pragma unroll
      for (int j = 0; j < H; ++j) {
        const bool there = at_of(tile, piece_block(j)) >= 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned bad = code_nans(vc[j][i]);
          mine_spoiled |= there && bad != 0;
          vc[j][i] = there ? vc[j][i] & ~bad : 0;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const int b = piece_block(j);
      // key operands: [32 tokens][16 channels][half of 8 channels][token]
#pragma unroll
      for (int e = 0; e < 2; ++e)
        keys[buf][(((b >> 1) * KK + half * 4 + g) * 2 + e) * 32 + (b & 1) * 16 + tok] = widen<BF16>(kc[j][2 * e], kc[j][2 * e + 1]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        reinterpret_cast<uint2 *>(values[buf])[value_at(j, i)] = make_uint2(Operand<false>::pair(vc[j][i], false), Operand<false>::pair(vc[j][i], true));
    }
  };

  f16v acc[OB];
#pragma unroll
  for (int o = 0; o < OB; ++o) acc[o] = f16v{0};
  Top top = {kLowest, kFirstE};
  float level = kLowest;                             // M less kBase, in one
  unsigned long long far = 0;                        // lanes whose M is beyond kNear (as a bool 587 us at 8192 tokens, 32 heads, so 571)
  float sum = 0;
  if (threadIdx.x == 0) spoiled = 0;
  if (from < to) {
    look(from);
    place(from);
    turn();
    look(from + kChunk);
    request(from);
    stage(from, from & 1);
    request(from + 1);
  }

  // A tile's 64 tokens are worked on as two halves: the scores of the second are multiplied while the weights of the first are
  // computed, and its weights while the first half's go into the values.
  bool whole, active;
  float f[4], add[4], units[4];
  f16v x[2];
  auto enter = [&](int tile) {
    const int i = (tile - chunk) * 4;
    whole = tile >= mine_first && tile < mine_last;
    active = have;
    if (!whole) {
      bool some = false;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int t0 = span.block(tile * 4 + b) * kBlock;
        some |= at_of(tile, b) >= 0 && t0 <= wave_hi && (c.window == 0 || t0 + kBlock + c.window > wave_lo || t0 < c.sinks);
      }
      active &= some;
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      f[b] = read_lane(factor, i + b);
      add[b] = read_lane(shift, i + b);
      units[b] = read_lane(unit, i + b);
    }
  };
  // The operands of a product are read from the LDS ahead of what comes before it, so that it does not wait (8192 tokens, 32 heads, a call
  // at a time: 624 us; with the first half of them ahead 631.  Each read as soon as the product before has used its registers: 628, and 657
  // with the barrier before a tile's last product, which then meets no wait for the LDS at all).
  static_assert(KK == 2 * OB, "as many operands of keys as of values");
  u4 ahead[KK];
  auto keys_ahead = [&](int buf, int m) {
#pragma unroll
    for (int k = 0; k < KK; ++k) ahead[k] = keys[buf][(m * KK + k) * 64 + lane];
  };
  auto values_ahead = [&](int buf, int m) {
#pragma unroll
    for (int o = 0; o < KK; ++o) ahead[o] = values[buf][(m * KK + o) * 64 + lane];
  };
  auto scores = [&](int m) {
    x[m] = f16v{0};
#pragma unroll
    for (int k = 0; k < KK; ++k) x[m] = Operand<BF16>::mma32(ahead[k], q[k], x[m]);
  };
  // Which of the lane's eight tokens of a block the row sees is a word of bits (four compares a score took 470
  // us at 40 heads, 4 x 4096 tokens, a window of 820, two 440, this 415).
  auto mask = [&](int tile, int m) {
    auto below = [](int n) { return (1u << min(max(n, 0), 12)) - 1; };
#pragma unroll
    for (int b = 2 * m; b < 2 * m + 2; ++b) {
      const int t0 = span.block(tile * 4 + b) * kBlock + 4 * h;        // the lane has t0 .. t0 + 3 and t0 + 8 .. t0 + 11
      unsigned seen = (below(p + 1 - t0) & ~below(from_token - t0)) | below(first_tokens - t0);
      if (at_of(tile, b) < 0) seen = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned all = (unsigned)((int)(seen << (31 - (i & 3) - 8 * (i >> 2))) >> 31);
        x[m][b % 2 * 8 + i] = __uint_as_float((__float_as_uint(x[m][b % 2 * 8 + i]) & all) | (0xff800000u & ~all));
      }
    }
  };
  // Weights of half m, and what they add to the sum (before 2^-e).  Whether one is too large for fp16 shows in these, so the maximum is
  // only looked for where one is, or where scores are far from 0: then M is moved and the weights are computed again, each step rounded by itself.
  u4 weights[2];
  float part[2];
  auto weigh = [&](int m) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float zero = add[2 * m + b] - level;
      part[b] = 0;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float y = exp2_fast(fmaf(x[m][b * 8 + i], f[2 * m + b], zero)), z = exp2_fast(fmaf(x[m][b * 8 + i + 1], f[2 * m + b], zero));
        part[b] += y + z;
        weights[b][i / 2] = half_pair(y, z);
      }
    }
  };
  auto weigh_exactly = [&](int m) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float factor = f[2 * m + b], e = add[2 * m + b] - top.e;
      part[b] = 0;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float y = exp2_fast((product(x[m][b * 8 + i], factor) - top.s) + e), z = exp2_fast((product(x[m][b * 8 + i + 1], factor) - top.s) + e);
        part[b] += y + z;
        weights[b][i / 2] = half_pair(y, z);
      }
    }
  };
  auto settle = [&](int m) {
    if (far | __ballot(fmaxf(part[0], part[1]) > kMost)) {
      Top most;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float y = x[m][b * 8];
#pragma unroll
        for (int i = 1; i < 8; ++i) y = fmaxf(y, x[m][b * 8 + i]);      // (the factor is positive)
        const float score = product(y, f[2 * m + b]), e = add[2 * m + b] - kBase;
        if (b == 0) most = Top{score, e};
        else most.raise(score, e);
      }
      most.raise_over<32>();
      const Top was = top;
      top.raise(most.s, most.e);
      const float less = exp2_fast(top.above(was.s, was.e));
      level = top.s + top.e;
      far = __ballot(fabsf(top.s) > kNear && top.s > kLowest);
      sum *= less;
#pragma unroll
      for (int o = 0; o < OB; ++o) acc[o] *= less;
      weigh_exactly(m);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) sum = fmaf(part[b], units[2 * m + b], sum);
  };
  auto gather = [&](const u4 (&w)[2]) {
#pragma unroll
    for (int o = 0; o < KK; ++o) acc[o % OB] = Operand<false>::mma32(ahead[o], w[o / OB], acc[o % OB]);
  };
#pragma unroll
  for (int k = 0; k < KK; ++k) asm volatile("" : "+v"(q[k]));          // the queries are waited for here, not (with all codes requested since) in the loop
  __syncthreads();
  if (from < to) {
    enter(from);
    if (active) {
      keys_ahead(from & 1, 0);
      scores(0);
      if (!whole) mask(from, 0);
    }
  }
  for (int tile = from; tile < to; ++tile) {
    const int buf = tile & 1;
    __builtin_amdgcn_s_setprio(0);
    keys_ahead(buf, 1);
    if (tile - chunk == kChunk / 2) place(chunk + kChunk);
    if (tile + 1 < to) {                             // (requested a round ago)
      stage(tile + 1, buf ^ 1);
      request(tile + 2);
    }
    if (active) {
      // products before the other workgroup's staging: 661 -> 621 us at 32 heads x 8192 tokens, clocks settled
      __builtin_amdgcn_s_setprio(1);
      scores(1);
      weigh(0);
      values_ahead(buf, 0);
      settle(0);
      if (!whole) mask(tile, 1);
      const u4 first[2] = {weights[0], weights[1]};
      gather(first);
      weigh(1);
      values_ahead(buf, 1);
      settle(1);
      gather(weights);
    }
    if (tile + 1 == to) break;
    if (tile + 1 - chunk == kChunk) {
      turn();
      chunk += kChunk;
      look(chunk + kChunk);
    }
    enter(tile + 1);
    __syncthreads();
    if (active) {
      keys_ahead(buf ^ 1, 0);
      scores(0);
      if (!whole) mask(tile + 1, 0);
    }
  }

  if (mine_spoiled) spoiled = 1;
  __syncthreads();
  if (spoiled)                                       // the NaN that were taken out, counted for the rows that see them
    for (int tile = from; tile < to; ++tile) {
      chunk = tile;
      look(tile);
      place(tile);
      at = at_next;
      if (tile >= all_first && tile < all_last) continue;
      request(tile);
#pragma unroll
      for (int j = 0; j < H; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned one = code_nans(vc[j][i]) & 0x38383838u;      // the code of 1
          reinterpret_cast<uint2 *>(values[0])[value_at(j, i)] = make_uint2(Operand<false>::pair(one, false), Operand<false>::pair(one, true));
        }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int t0 = span.block(tile * 4 + b) * kBlock;
        half8 seen;
#pragma unroll
        for (int i = 0; i < 8; ++i) seen[i] = at_of(tile, b) >= 0 && sees(c, p, t0 + (i & 3) + 4 * h + 8 * (i >> 2)) ? 1 : 0;
#pragma unroll
        for (int o = 0; o < OB; ++o) {
          const f16v count = Operand<false>::mma32(values[0][(b * OB + o) * 64 + lane], __builtin_bit_cast(u4, seen), f16v{0});
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[o][i] = count[i] > 0 ? __builtin_nanf("") : acc[o][i];
        }
      }
      __syncthreads();
    }

  sum += __shfl_xor(sum, 32, kWave);
  if constexpr (kTrunk) {
    if (col > last_col) return;
    const long in_head = trunk.node.base + (long)trunk.piece * trunk.node.cols + col, at = head * a.columns + in_head;
    if (trunk.node.base < 0 || in_head >= a.columns) return;
    const float unit_of_e = top.unit();
    if (from < to)
#pragma unroll
      for (int o = 0; o < OB; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f4 *>(a.trunk + at * D + o * 32 + i * 8 + h * 4) =
              f4{acc[o][4 * i], acc[o][4 * i + 1], acc[o][4 * i + 2], acc[o][4 * i + 3]} * unit_of_e;
    if (h == 0) {
      float *tops = a.trunk + c.heads * a.columns * D;
      tops[at] = from < to ? top.s : -__builtin_inff();
      if (trunk.only && in_head + trunk.node.cols < a.columns) tops[at + trunk.node.cols] = -__builtin_inff();
      tops[c.heads * a.columns + at] = sum * unit_of_e;
    }
    return;
  }
  if (splits > 1) {
    float *share = a.parts + few_floats(G, D) + (long)id * wide_floats(D);
    const int mine = wave * 32 + n;
    const float unit_of_e = top.unit();
    if (from < to)
#pragma unroll
      for (int o = 0; o < OB; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f4 *>(share + mine * D + o * 32 + i * 8 + h * 4) =
              f4{acc[o][4 * i], acc[o][4 * i + 1], acc[o][4 * i + 2], acc[o][4 * i + 3]} * unit_of_e;
    if (h == 0) { share[kWide * D + mine] = from < to ? top.s : -__builtin_inff(); share[kWide * (D + 1) + mine] = sum * unit_of_e; }
    return;
  }
  if (col > last_col) return;
  const float r = 1.f / sum;
  const long to_row = (long)row * c.heads * G + q_head;
#pragma unroll
  for (int o = 0; o < OB; ++o)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      auto stored = [&](int j) { return (unsigned)Operand<BF16>::store(share_of(acc[o][4 * i + j], sum, r)); };
      const uint2 y = make_uint2(stored(0) | stored(1) << 16, stored(2) | stored(3) << 16);
      reinterpret_cast<uint2 *>(a.out)[to_row * (D / 4) + o * 8 + i * 2 + h] = y;
    }
  if (a.lse && h == 0) a.lse[to_row] = sum == 0.f ? -__builtin_inff() : (top.s + (top.e + __builtin_log2f(sum))) * 0.6931471805599453f;
