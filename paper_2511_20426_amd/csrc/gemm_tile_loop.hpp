// The main loop of a compiled tile, included in the bodies of the kernels that have one (a function of its own gave the plain
// products' kernels other registers): K walked in stages of 128 bytes of a row through a ring in LDS.  Uses T (the TileShape),
// kStages, BN, Products (the types and the matrix instruction), lds, wave, wm, wn, l15, grp, n_stages, and base_w, base_x, offw, offx: where
// the lane's part of the loads starts.  Leaves the sums in acc, the ring free.
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
  int issued = 0;
  uint32_t fill = lds0;                       // ring slot the next stage goes to
  auto issue = [&]() {
#pragma unroll
    for (int i = 0; i < T::kLoadsW; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :: "s"(fill + (wave * T::kLoadsW + i) * 1024), "v"(offw[i]), "s"(base_w) : "memory", "m0");
#pragma unroll
    for (int i = 0; i < T::kLoadsX; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :: "s"(fill + BN * 128 + (wave * T::kLoadsX + i) * 1024), "v"(offx[i]), "s"(base_x) : "memory", "m0");
    // past the last stage the loads repeat it, into slots nothing reads any more: the wait counts stay exact
    ++issued;
    base_w += issued < n_stages ? 128 : 0;
    base_x += issued < n_stages ? 128 : 0;
    fill += T::kStageBytes;
    fill = fill == lds0 + kStages * T::kStageBytes ? lds0 : fill;
  };
  const uint32_t swz = (l15 >> 1) & 7;
  const uint32_t aw0 = uint32_t((wn * T::kTn * 16 + l15) * 128) + ((uint32_t(grp) ^ swz) << 4);
  const uint32_t ax0 = uint32_t(BN * 128 + (wm * T::kTm * 16 + l15) * 128) + ((uint32_t(grp) ^ swz) << 4);

  typename Products::Sums acc[T::kTn][T::kTm];
#pragma unroll
  for (int i = 0; i < T::kTn; ++i)
#pragma unroll
    for (int j = 0; j < T::kTm; ++j) acc[i][j] = typename Products::Sums{0, 0, 0, 0};
  typename Products::Frag fw[2][T::kTn], fx[2][T::kTm];
  uint32_t slot = 0;
  auto read = [&](int kk) {
#pragma unroll
    for (int i = 0; i < T::kTn; ++i) fw[kk][i] = *reinterpret_cast<const typename Products::Frag*>(lds + slot + (aw0 ^ (kk << 6)) + i * 2048);
#pragma unroll
    for (int j = 0; j < T::kTm; ++j) fx[kk][j] = *reinterpret_cast<const typename Products::Frag*>(lds + slot + (ax0 ^ (kk << 6)) + j * 2048);
    __builtin_amdgcn_sched_barrier(0);        // reads stay ahead of the products they run beside
  };
  auto multiply = [&](int kk) {
#pragma unroll
    for (int i = 0; i < T::kTn; ++i)
#pragma unroll
      for (int j = 0; j < T::kTm; ++j) acc[i][j] = Products::multiply(fw[kk][i], fx[kk][j], acc[i][j]);
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) issue();
  constexpr int kFlying = (kStages - 1) * (T::kLoadsW + T::kLoadsX);
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"(kFlying) : "memory");
  read(0);
  // operands are read one k-step ahead of their products, across stages too: the barrier stands before a
  // stage's second k-step
  for (int s = 0; s < n_stages; ++s) {
    read(1);
    multiply(0);
    __builtin_amdgcn_sched_barrier(0);
    // the next stage has landed; every wave has this one in registers: its slot takes the next loads
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(kFlying - T::kLoadsW - T::kLoadsX) : "memory");
    issue();
    slot += T::kStageBytes;
    slot = slot == kStages * T::kStageBytes ? 0 : slot;
    read(0);
    multiply(1);
    __builtin_amdgcn_sched_barrier(0);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");     // the ring is free
