// What the entry points of all sources share: the state of the last call on this host thread (api.cu).
#pragma once

namespace xconv {

extern thread_local int g_last_cuda_error, g_launches;
void new_call();               // a fresh tag, no launches
unsigned int call_tag();

}  // namespace xconv
